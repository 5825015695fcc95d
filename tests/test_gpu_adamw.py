"""The AdamW step over many tensors.  32-bit states and parameters against the formulas in 64 bits; 8-bit states bit for bit against their
definition, carried out in numpy's fp32 (every operation of it rounds once), and against the law of their chances.

With u = 2^-24: m is a sum of two products whose factors are rounded: 3 u (|b1 m| + |c1 g|); v the same with one product more, all of one
sign: 5 u v; r = sqrt(v): 4 u r; root r + eps: 8 u of itself; m / that: 9 u of itself and the error of m; times size, taken from
keep p: 3 u |keep p| + 12 u |change| + size / (root r + eps) times the error of m; and half a step of the parameter's type."""
import math

import numpy as np
import pytest

from paper_2506_22714_amd import binding as lb

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

U = 2.0 ** -24
TYPES = [torch.float16, torch.bfloat16, torch.float32]
SMALLEST = {torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134, torch.float32: 2.0 ** -149}
E4M3 = np.array([(-1) ** (c >> 7) * (np.nan if c & 127 == 127 else (c & 7) * 2.0 ** -9 if not c & 120 else (8 + (c & 7)) * 2.0 ** ((c >> 3 & 15) - 10))
                 for c in range(256)])
HYPER = dict(lr=2e-3, betas=(0.9, 0.99), eps=1e-8, weight_decay=0.03)


@pytest.fixture(scope="module", autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    lb.lib()


# ---- the definition of 8-bit states ----
def mix(x):
    x = np.asarray(x, dtype=np.uint32)
    x = x ^ (x >> np.uint32(16))
    x = x * np.uint32(0x6C8E9CF5)
    x = x ^ (x >> np.uint32(15))
    x = x * np.uint32(0x58AC4D6B)
    return x ^ (x >> np.uint32(16))


def chances(n, seed, step, number, begin=0):
    with np.errstate(over="ignore"):
        key = mix(mix(mix(np.uint32(seed)) + np.uint32(step)) + np.uint32(number))
        i = np.arange(begin, begin + n, dtype=np.uint64)
        h = mix(key + (i & np.uint64(0xffffffff)).astype(np.uint32) + (i >> np.uint64(32)).astype(np.uint32) * np.uint32(0x9E3779B1))
    return (h & np.uint32(0xffff)).astype(np.float32) * np.float32(2.0 ** -16), (h >> np.uint32(16)).astype(np.float32) * np.float32(2.0 ** -16)


def encode(x, chance, root):
    x = np.asarray(x, dtype=np.float32)
    n = x.size
    a = np.abs(x).astype(np.float32)
    known = np.where(np.isfinite(a), a, np.float32(0))
    most = np.pad(known, (0, -n % 256)).reshape(-1, 256).max(1)
    scales = np.empty(most.size, dtype=np.float32)
    for k, v in enumerate(most):
        e = -126
        while float(v) > 448.0 * 2.0 ** e:
            e += 1
        scales[k] = 2.0 ** e
    y = (a / np.repeat(scales, 256)[:n]).astype(np.float32)
    with np.errstate(invalid="ignore", divide="ignore"):
        e = np.maximum(np.where((y > 0) & np.isfinite(y), np.frexp(np.where(np.isfinite(y), y, 1))[1] - 1, -6), -6)
        q = np.floor((y * np.exp2(3.0 - e).astype(np.float32) + chance).astype(np.float32))
    if root:
        q = np.where((x > 0) & (q == 0), 1, q)
    code = np.where(np.isfinite(y), 8 * (e + 6) + np.where(np.isfinite(q), q, 0), 127).astype(np.uint8)
    return code if root else code | (np.signbit(x).astype(np.uint8) << 7), scales


def decode(codes, scales):
    return (E4M3[codes] * np.repeat(scales, 256)[:codes.size]).astype(np.float32)


def states_after(m, v, g, betas):
    """m, v, sqrt(v) after the step in fp32, an operation at a time."""
    b1, b2 = (np.float32(b) for b in betas)
    c1, c2 = (np.float32(1 - b) for b in betas)
    m = b1 * m + c1 * g
    v = b2 * v + c2 * (g * g)
    return m, v, np.sqrt(v)


def check_parameter(got, p, g, m, v, step, dtype, h=HYPER):
    p, g, m, v = (np.asarray(t, dtype=np.float64) for t in (p, g, m, v))
    b1, b2 = h["betas"]
    dm = 3 * U * (np.abs(b1 * m) + np.abs((1 - b1) * g)) + 2.0 ** -149
    m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    den = np.sqrt(v / (1 - b2 ** step)) + h["eps"]
    # (squares below the smallest fp32 numbers are rounded to multiples of them: the root is off by that much where it is that small)
    small = 2.0 ** -74 / math.sqrt(1 - b2 ** step) / den
    size = h["lr"] / (1 - b1 ** step)
    keep = 1 - h["lr"] * h["weight_decay"]
    ref = keep * p - size * m / den
    tol = 3 * U * np.abs(keep * p) + (12 * U + small) * np.abs(size * m / den) + size / den * dm
    tol = tol + torch.finfo(dtype).eps / 2 * np.abs(ref) * (1 + 2.0 ** -8) + SMALLEST[dtype]
    far = np.abs(got.detach().double().cpu().numpy().reshape(-1) - ref) - tol
    assert far.max() <= 0, (float(far.max()), int(far.argmax()))
    return m, v


class Model:
    """Lists of tensors as a program has them, with copies on the host."""

    def __init__(self, sizes, dtype, bits, master, seed=0, offset=0):
        rng = np.random.default_rng(seed)
        place = lambda a, t: torch.cat([torch.zeros(offset), torch.from_numpy(a).reshape(-1)]).to(t).cuda()[offset:]      # noqa: E731
        self.params, self.grads, self.first, self.second, self.masters, self.fs, self.ss = [], [], [], [], [], [], []
        for n in sizes:
            self.masters.append(place(rng.standard_normal(n).astype(np.float32), torch.float32))
            self.params.append(place(self.masters[-1].cpu().numpy(), dtype))
            size = 10.0 ** rng.uniform(-4, 1)
            g = size * rng.standard_normal(n)
            self.grads.append(place(np.where(rng.random(n) < 0.2, 0, g).astype(np.float32), dtype))
            m = (0.5 * size * rng.standard_normal(n) * 10 ** rng.uniform(-3, 0, n)).astype(np.float32)
            r = (size * 10 ** rng.uniform(-4, 0, n)).astype(np.float32)
            if bits == 8:
                for x, codes, scales, root in ((m, self.first, self.fs, False), (r, self.second, self.ss, True)):
                    c, s = encode(x, np.full(n, 0.5, dtype=np.float32), root)
                    codes.append(torch.cat([torch.zeros(offset, dtype=torch.uint8), torch.from_numpy(c)]).cuda()[offset:].view(torch.float8_e4m3fn))
                    scales.append(torch.from_numpy(s).cuda())
            else:
                self.first.append(place(m, torch.float32))
                self.second.append(place(r * r, torch.float32))
        self.bits, self.dtype, self.master = bits, dtype, master

    def step(self, step, seed=0, **kw):
        lb.adamw(self.params, self.grads, self.first, self.second, step, **{**HYPER, **kw}, first_scales=self.fs if self.bits == 8 else None,
                 second_scales=self.ss if self.bits == 8 else None, masters=self.masters if self.master else None, seed=seed)

    def host(self, k):
        """(p, g, m, v) in fp32, as they are now."""
        p = (self.masters[k] if self.master else self.params[k].float()).cpu().numpy()
        g = self.grads[k].float().cpu().numpy()
        if self.bits == 8:
            m, r = (decode(c[k].view(torch.uint8).cpu().numpy(), s[k].cpu().numpy()) for c, s in ((self.first, self.fs), (self.second, self.ss)))
            return p, g, m, r * r
        return p, g, self.first[k].cpu().numpy(), self.second[k].cpu().numpy()

    def checked_step(self, step, seed=0, numbers=None):
        before = [self.host(k) for k in range(len(self.params))]
        self.step(step, seed)
        for k, (p, g, m, v) in enumerate(before):
            if p.size == 0:
                continue
            check_parameter(self.masters[k] if self.master else self.params[k], p, g, m, v, step, torch.float32 if self.master else self.dtype)
            if self.master:
                assert torch.equal(self.params[k], self.masters[k].to(self.dtype))
            m, v, r = states_after(m, v, g, HYPER["betas"])
            if self.bits == 32:
                np.testing.assert_array_equal(self.first[k].cpu().numpy(), m)
                np.testing.assert_array_equal(self.second[k].cpu().numpy(), v)
                continue
            chance = chances(p.size, seed, step, k if numbers is None else numbers[k])
            for got, scales, want in ((self.first[k], self.fs[k], encode(m, chance[0], False)), (self.second[k], self.ss[k], encode(r, chance[1], True))):
                np.testing.assert_array_equal(scales.cpu().numpy(), want[1])
                np.testing.assert_array_equal(got.view(torch.uint8).cpu().numpy(), want[0])


def test_torch_reads_the_codes_as_the_definition_does():
    np.testing.assert_array_equal(torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy(), E4M3.astype(np.float32))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("master", [False, True])
def test_steps(dtype, bits, master):
    model = Model([1, 2, 255, 256, 257, 64 * 64, 64, 1000, 0, 4096, 4097, 77777], dtype, bits, master, seed=bits)
    for step in (1, 2, 3, 1000):
        model.checked_step(step, seed=step * 77)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("offset", [1, 3, 4, 8])
def test_tensors_that_begin_anywhere(dtype, bits, offset):
    model = Model([5, 300, 8193, 20000], dtype, bits, dtype != torch.float32, seed=offset, offset=offset)
    keep = [t._base.view(torch.uint8)[: offset * t.element_size()].clone() for t in model.params if t._base is not None]
    model.checked_step(1)
    model.checked_step(2)
    for t, k in zip([t for t in model.params if t._base is not None], keep):
        assert torch.equal(t._base.view(torch.uint8)[: k.numel()], k)


@pytest.mark.parametrize("bits", [32, 8])
def test_more_tensors_than_a_launch_takes_and_all_types_at_once(bits):
    rng = np.random.default_rng(0)
    models = [Model(rng.integers(1, 3000, 45).tolist(), t, bits, False, seed=7) for t in TYPES]
    alone = [Model([p.numel() for p in m.params], m.dtype, bits, False, seed=7) for m in models]
    order = rng.permutation(135)
    pick = lambda name: [getattr(models[k // 45], name)[k % 45] for k in order]      # noqa: E731
    numbers = [int(k) for k in order]
    lb.adamw(pick("params"), pick("grads"), pick("first"), pick("second"), 3, **HYPER, first_scales=pick("fs") if bits == 8 else None,
             second_scales=pick("ss") if bits == 8 else None, numbers=numbers, seed=5)
    for j, m in enumerate(alone):
        lb.adamw(m.params, m.grads, m.first, m.second, 3, **HYPER, first_scales=m.fs if bits == 8 else None,
                 second_scales=m.ss if bits == 8 else None, numbers=[45 * j + k for k in range(45)], seed=5)
        for name in ("params", "first", "second", "fs", "ss"):
            for a, b in zip(getattr(models[j], name), getattr(m, name)):
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_special_numbers_in_8_bits():
    """Zeros stay zeros, the tiny and the huge, an Inf and a NaN spoil their own element alone, a root above zero stays above zero."""
    n = 256 * 6
    m = Model([n], torch.float32, 8, False)
    g = torch.zeros(n, device="cuda")
    g[256:512] = 1e-30                              # squares vanish
    g[512:768] = 1e18
    g[768] = float("inf")
    g[769] = float("nan")
    g[770:1024] = 0.5
    g[1024] = 1e-6                                  # beside numbers a million times as large
    g[1025:1280] = 1.0
    g[1280:] = 2.0 ** -64
    m.grads[0] = g
    for t in (m.first[0], m.second[0]):
        t.view(torch.uint8).zero_()
    p, _, m0, v0 = m.host(0)
    m.step(1, seed=3)
    after = states_after(m0, v0, g.cpu().numpy(), HYPER["betas"])
    chance = chances(n, 3, 1, 0)
    for got, scales, x, c, root in ((m.first[0], m.fs[0], after[0], chance[0], False), (m.second[0], m.ss[0], after[2], chance[1], True)):
        code, s = encode(x, c, root)
        np.testing.assert_array_equal(scales.cpu().numpy(), s)
        np.testing.assert_array_equal(got.view(torch.uint8).cpu().numpy(), code)
    first, second = m.first[0].float(), m.second[0].float()
    assert bool((first[:256] == 0).all()) and bool((second[:256] == 0).all())
    assert bool(first[768:770].isnan().all()) and bool(second[768:770].isnan().all()) and bool(first[770:].isfinite().all())
    assert bool((second[770:] > 0).all()) and float(second[1024]) == 2.0 ** -9
    assert bool(m.params[0][:768].isfinite().all()) and bool(m.params[0][770:].isfinite().all())


def test_chances_follow_the_distance():
    """2^20 elements of one value between two neighbours: the share that goes up is the distance to the lower one, within five standard
    deviations; another step, seed or tensor draws other chances."""
    n = 1 << 20
    x = 1.3                                         # m = c1 g: between 1.25 and 1.375 in blocks whose largest is 448
    def one(step, seed, numbers=None):
        g = torch.full((n,), x, device="cuda")
        g[::256] = 448.0
        first, second = (torch.zeros(n, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
        scales = [torch.ones(n // 256, device="cuda") for _ in range(2)]
        lb.adamw([torch.zeros(n, device="cuda")], [g], [first], [second], step, lr=0.0, betas=(0.0, 0.0), first_scales=[scales[0]],
                 second_scales=[scales[1]], seed=seed, numbers=numbers)
        keep = torch.ones(n, dtype=torch.bool, device="cuda")
        keep[::256] = False
        return first.float()[keep], second.float()[keep]
    seen = []
    for args in ((1, 0), (2, 0), (1, 1), (1, 0, [1])):
        for y in one(*args):
            assert bool(((y == 1.25) | (y == 1.375)).all())
            share = float((y == 1.375).double().mean())
            want = (x - 1.25) / 0.125
            assert abs(share - want) < 5 * math.sqrt(want * (1 - want) / y.numel()) + 2.0 ** -15
            seen.append(y == 1.375)
    for a in range(len(seen)):
        for b in range(a):
            both = float((seen[a] & seen[b]).double().mean())
            assert abs(both - want * want) < 5 * math.sqrt(want ** 2 * (1 - want ** 2) / seen[a].numel()) + 2.0 ** -14


def test_averages_move_in_8_bits():
    """A gradient of constant size drives sqrt(v) to that size though each step is far below the distance of two codes."""
    n = 1 << 14
    g = torch.full((n,), 0.5, device="cuda")
    p = torch.zeros(n, device="cuda")
    codes = [torch.zeros(n, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2)]
    scales = [torch.ones(n // 256, device="cuda") for _ in range(2)]
    for step in range(1, 2001):
        lb.adamw([p], [g], [codes[0]], [codes[1]], step, lr=0.0, betas=(0.9, 0.999), first_scales=[scales[0]], second_scales=[scales[1]])
    r = codes[1].float() * scales[1].repeat_interleave(256)
    # v = 0.25 (1 - 0.999^2000), and as much again at most: each rounding of r adds its variance, (r / 8)^2 / 4 at most, to v, a thousandth of which stays ...
    want = 0.5 * math.sqrt(1 - 0.999 ** 2000)
    mean = float(r.double().mean())
    assert 0.8 * want < mean < 1.25 * want
    assert abs(float((codes[0].float() * scales[0].repeat_interleave(256)).double().mean()) - 0.5) < 0.01


def test_step_and_rate_on_the_gpu_and_replayed():
    sizes = [300, 70000, 5]
    for bits in (32, 8):
        a, b = Model(sizes, torch.bfloat16, bits, True, seed=1), Model(sizes, torch.bfloat16, bits, True, seed=1)
        step, lr = torch.zeros((), dtype=torch.int64, device="cuda"), torch.full((1,), 1e-3, device="cuda")
        graph = torch.cuda.CUDAGraph()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            lb.lib()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            step += 1
            a.step(step, seed=9, lr=lr)
        for k in range(1, 5):
            lr.fill_(k * 1e-3)
            for x in a.grads:
                x.normal_()
            for x, y in zip(b.grads, a.grads):
                x.copy_(y)
            graph.replay()
            b.step(k, seed=9, lr=float(lr))
            torch.cuda.synchronize()
            for x, y in zip(a.first + a.second + a.fs + a.ss, b.first + b.second + b.fs + b.ss):
                assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
            for x, y in zip(a.masters, b.masters):
                # the rate per step is made by expm1 and pow: rounded to fp32 it may differ in its last place
                assert float((x - y).abs().max()) <= 4 * 2.0 ** -23 * k * 1e-3 * 20 + 2 * 2.0 ** -24 * float(y.abs().max()) * k


def test_offsets_beyond_32_bits():
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs some 45 GiB")
    n = (1 << 32) + 300
    p, g = torch.zeros(n, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    first, second = (torch.zeros(n, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
    scales = [torch.ones(-(-n // 256), device="cuda") for _ in range(2)]
    tail = torch.randn(1000, device="cuda").bfloat16()
    g[-1000:] = tail
    lb.adamw([p], [g], [first], [second], 1, **HYPER, first_scales=[scales[0]], second_scales=[scales[1]], seed=4)
    begin = n - 1000
    lead = begin % 256
    x = np.concatenate([np.zeros(lead, dtype=np.float32), tail.float().cpu().numpy()])
    zero = np.zeros_like(x)
    m, v, r = states_after(zero, zero, x, HYPER["betas"])
    chance = chances(x.size, 4, 1, 0, begin - lead)
    for got, s, want in ((first, scales[0], encode(m, chance[0], False)), (second, scales[1], encode(r, chance[1], True))):
        np.testing.assert_array_equal(got.view(torch.uint8)[begin - lead:].cpu().numpy(), want[0])
        np.testing.assert_array_equal(s[(begin - lead) // 256:].cpu().numpy(), want[1])
    check_parameter(p[begin - lead:], zero, x, zero, zero, 1, torch.bfloat16)
    assert not bool(p[: begin - lead].any())
    del p, g, first, second
    torch.cuda.empty_cache()


def test_a_graph_that_saved_a_parameter_notices_the_step():
    p = torch.ones(5, device="cuda", requires_grad=True)
    loss = (p * p).sum()
    s = [torch.zeros(5, device="cuda") for _ in range(2)]
    lb.adamw([p], [torch.ones(5, device="cuda")], [s[0]], [s[1]], 1)
    with pytest.raises(RuntimeError):
        loss.backward()


def test_refusals_of_the_binding():
    x = lambda *s, **k: torch.zeros(*s, device="cuda", **k)       # noqa: E731
    p, f = [x(8)], [x(8)]
    codes = [x(8).to(torch.float8_e4m3fn)]
    for call in (lambda: lb.adamw(p, [x(7)], f, [x(8)], 1), lambda: lb.adamw(p, [x(8).half()], f, [x(8)], 1), lambda: lb.adamw(p, [x(16)[::2]], f, [x(8)], 1),
                 lambda: lb.adamw(p, f, [x(8).half()], [x(8)], 1), lambda: lb.adamw(p, f, codes, codes, 1), lambda: lb.adamw(p, f, p, f, 1, first_scales=[x(1)], second_scales=[x(1)]),
                 lambda: lb.adamw(p, f, codes, codes, 1, first_scales=[x(2)], second_scales=[x(1)]), lambda: lb.adamw(p * 2, f * 2, f * 2, f * 2, 1),
                 lambda: lb.adamw(p, f, f, f, torch.ones(1, device="cuda")), lambda: lb.adamw(p, f, f, f, 1, lr=torch.ones(1)), lambda: lb.adamw([p[0].double()], f, f, f, 1),
                 lambda: lb.adamw(p, f, f, f, 1, masters=[x(8).half()])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(lb.LibraError):
        lb.adamw(p, f, [x(8)], [x(8)], 0)


# ---- the optimizer ----
def test_optimizer_against_the_call():
    from paper_2506_22714_amd.optim import AdamW
    for bits in (32, 8):
        ps = [torch.nn.Parameter(torch.randn(*s, device="cuda").bfloat16()) for s in ((30, 40), (7,), (500,))]
        opt = AdamW([{"params": ps[:2]}, {"params": ps[2:], "lr": 0.01}], **HYPER, state_bits=bits, master=True, seed=6)
        masters = [p.detach().float() for p in ps]
        new = lambda p: torch.zeros_like(p, dtype=torch.float32) if bits == 32 else torch.zeros(p.shape, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)    # noqa: E731
        first, second = [new(p) for p in ps], [new(p) for p in ps]
        scales = [[torch.ones(-(-p.numel() // 256), device="cuda") for p in ps] for _ in range(2)]
        steps, copies = [0, 0, 0], [p.detach().clone() for p in ps]
        for t in range(4):
            for k, p in enumerate(ps):
                p.grad = torch.randn_like(p) if not (k == 1 and t == 1) else None
            for k, p in enumerate(ps):
                if p.grad is None:
                    continue
                steps[k] += 1
                lb.adamw([copies[k]], [p.grad], [first[k]], [second[k]], steps[k], **{**HYPER, **({"lr": 0.01} if k == 2 else {})}, seed=6, numbers=[k],
                         masters=[masters[k]], first_scales=[scales[0][k]] if bits == 8 else None, second_scales=[scales[1][k]] if bits == 8 else None)
            opt.step()
            if t == 2:                                            # leaves and comes back with its states
                again = AdamW([{"params": ps[:2]}, {"params": ps[2:]}], state_bits=bits, master=True)
                again.load_state_dict(opt.state_dict())
                opt = again
            for p, c in zip(ps, copies):
                assert torch.equal(p.detach(), c)
            for k, p in enumerate(ps):
                s = opt.state[p]
                assert s["step"] == steps[k] and torch.equal(s["master"], masters[k])
                assert torch.equal(s["first"].view(torch.uint8), first[k].view(torch.uint8)) and torch.equal(s["second"].view(torch.uint8), second[k].view(torch.uint8))


def test_optimizer_under_capture():
    from paper_2506_22714_amd.optim import AdamW
    make = lambda: [torch.nn.Parameter(torch.arange(600, dtype=torch.float32, device="cuda") / 600), torch.nn.Parameter(torch.ones(3, device="cuda"))]     # noqa: E731
    a, b = make(), make()
    for ps in (a, b):
        for p in ps:
            p.grad = torch.ones_like(p)
    lr = torch.full((1,), 1e-3, device="cuda")
    oa, ob = AdamW(a, lr=lr, state_bits=8, capturable=True), AdamW(b, lr=1e-3, state_bits=8)
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(RuntimeError, match="before the capture"):
        with torch.cuda.graph(graph):
            oa.step()
    torch.cuda.synchronize()
    oa.step()
    ob.step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        oa.step()
    for k in range(3):
        for x, y in zip(a, b):
            x.grad.normal_()
            y.grad.copy_(x.grad)
        lr.fill_(1e-3 * (k + 1))
        ob.param_groups[0]["lr"] = float(lr)
        graph.replay()
        ob.step()
        torch.cuda.synchronize()
        assert int(oa.param_groups[0]["step"]) == k + 2
        for x, y in zip(a, b):
            assert torch.equal(oa.state[x]["first"].view(torch.uint8), ob.state[y]["first"].view(torch.uint8))
            assert float((x - y).abs().max()) < 1e-6


@pytest.mark.parametrize("capturable", [False, True])
@pytest.mark.parametrize("bits", [32, 8])
def test_a_refused_step_counts_for_nothing(bits, capturable):
    """Whatever is refused, in whichever group: no parameter, state or count has changed, and the steps after it are what they would have been."""
    from paper_2506_22714_amd.optim import AdamW
    def make():
        ps = [torch.nn.Parameter(torch.linspace(-1, 1, n, device="cuda")) for n in (300, 7, 40)]
        return ps, AdamW([{"params": ps[:2]}, {"params": ps[2:], "lr": 1e-2}], lr=1e-3, state_bits=bits, capturable=capturable, seed=3)
    (ps, opt), (qs, plain) = make(), make()
    odd = torch.nn.Parameter(torch.ones(4, device="cuda", dtype=torch.float64))          # no type of the kernels
    opt.add_param_group({"params": [odd]})
    g = torch.Generator(device="cuda").manual_seed(0)
    for step in range(3):
        for p, q in zip(ps, qs):
            p.grad = torch.randn(p.shape, generator=g, device="cuda")
            q.grad = p.grad.clone()
        before = [p.detach().clone() for p in ps]
        odd.grad = torch.ones_like(odd)
        with pytest.raises(ValueError):
            opt.step()
        odd.grad = None
        for name, bad in (("lr", float("nan")), ("eps", float("nan")), ("betas", (0.9, 1.0))):
            good, opt.param_groups[1][name] = opt.param_groups[1][name], bad
            with pytest.raises(lb.LibraError):
                opt.step()
            opt.param_groups[1][name] = good
        assert all(torch.equal(p, b) for p, b in zip(ps, before))
        assert len(opt.state) == (3 if step else 0)
        opt.step()
        plain.step()
        for p, q in zip(ps, qs):
            assert torch.equal(p, q)
            a, b = opt.state[p], plain.state[q]
            assert a.get("step") == b.get("step") == (None if capturable else step + 1)
            for name in ("first", "second"):
                assert torch.equal(a[name].view(torch.uint8), b[name].view(torch.uint8))
        if capturable:
            assert [int(group["step"]) for group in opt.param_groups[:2]] == [step + 1] * 2


@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_that_counts_on_the_host_is_not_captured(bits):
    """Its number would be the same in every replay."""
    from paper_2506_22714_amd.optim import AdamW
    p, q = (torch.nn.Parameter(torch.ones(300, device="cuda")) for _ in range(2))
    p.grad, q.grad = torch.ones_like(p), torch.ones_like(q)
    opt = AdamW([{"params": [q], "capturable": True}, {"params": [p]}], state_bits=bits)
    opt.step()
    before = p.detach().clone(), q.detach().clone()
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(RuntimeError, match="capturable"):
        with torch.cuda.graph(graph):
            opt.step()
    torch.cuda.synchronize()
    assert opt.state[p]["step"] == 1 and int(opt.param_groups[0]["step"]) == 1
    assert torch.equal(p, before[0]) and torch.equal(q, before[1])
    opt.step()
    assert opt.state[p]["step"] == 2


@pytest.mark.parametrize("handle", [True, False])
@pytest.mark.parametrize("bits", [32, 8])
def test_a_checkpoint_on_the_cpu_goes_on(bits, handle):
    """Step numbers and rates on the GPU, saved, loaded to the CPU and from there into another optimizer: its steps are those of the first one.
    A rate that the program holds is filled, and read."""
    import io
    from paper_2506_22714_amd.optim import AdamW
    def make(lr):
        ps = [torch.nn.Parameter(torch.linspace(-1, 1, n, device="cuda").bfloat16()) for n in (300, 7)]
        return ps, AdamW([{"params": ps[:1]}, {"params": ps[1:], "lr": 5e-3}], lr=lr, state_bits=bits, master=True, capturable=True, seed=2)
    lr = torch.full((1,), 1e-2, device="cuda")
    ps, opt = make(lr)
    g = torch.Generator(device="cuda").manual_seed(1)
    def grads(*several):
        for k, n in enumerate((300, 7)):
            d = torch.randn(n, generator=g, device="cuda").bfloat16()
            for s in several:
                s[k].grad = d.clone()
    for _ in range(2):
        grads(ps)
        opt.step()
    file = io.BytesIO()
    torch.save(opt.state_dict(), file)
    file.seek(0)
    other = torch.zeros((), device="cuda") if handle else 0.5
    qs, again = make(other)
    again.load_state_dict(torch.load(file, map_location="cpu", weights_only=True))
    for p, q in zip(ps, qs):
        q.data.copy_(p.data)
    if handle:
        assert again.param_groups[0]["lr"] is other and float(other) == float(lr)
    assert again.param_groups[0]["lr"].device == ps[0].device and again.param_groups[1]["lr"] == 5e-3
    for k in range(3):
        if k == 1:
            lr.fill_(3e-2)
            again.param_groups[0]["lr"].fill_(3e-2)
        grads(ps, qs)
        opt.step()
        again.step()
        assert [int(x["step"]) for x in again.param_groups] == [k + 3] * 2
        for p, q in zip(ps, qs):
            assert torch.equal(p, q)
            for name, x in opt.state[p].items():
                assert torch.equal(x.view(torch.uint8), again.state[q][name].view(torch.uint8))


def test_rates_that_groups_share():
    """Two groups with one tensor take rates that differ apart."""
    from paper_2506_22714_amd.optim import AdamW
    make = lambda a, b: AdamW([{"params": [torch.nn.Parameter(torch.ones(3, device="cuda"))], "lr": x} for x in (a, b)], capturable=True)      # noqa: E731
    rate = lambda x: torch.full((1,), x, device="cuda")       # noqa: E731
    for want in ((1e-2, 1e-2), (1e-2, 2e-2)):
        shared = rate(5.0)
        opt = make(shared, shared)
        opt.load_state_dict(make(rate(want[0]), rate(want[1])).state_dict())
        assert [float(g["lr"]) for g in opt.param_groups] == [float(torch.tensor(x)) for x in want]
        assert opt.param_groups[0]["lr"] is shared and (opt.param_groups[1]["lr"] is shared) == (want[0] == want[1])


@pytest.mark.parametrize("bits", [32, 8])
def test_arrays_beside_each_other_and_shared_gradients(bits):
    """Parameters and states cut from one array each, without space between; a gradient that two parameters have; an fp32 copy that is its
    parameter.  What is written may not lie on anything else."""
    n = [256, 300, 20, 5000]
    at = np.concatenate([[0], np.cumsum(n)])
    def make(apart):
        cut = lambda t: [t[a:b].clone() if apart else t[a:b] for a, b in zip(at, at[1:])]      # noqa: E731
        f = lambda seed: torch.randn(int(at[-1]), generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")      # noqa: E731
        p = cut(f(0))
        g = f(1)
        grads = [g[:k] for k in n]                # all begin at one address
        if bits == 8:
            states = [[x.to(torch.float8_e4m3fn) for x in cut(f(2))], [x.to(torch.float8_e4m3fn) for x in cut(f(3).abs())]]
            return p, grads, *states, *[[torch.ones(-(-k // 256), device="cuda") for k in n] for _ in range(2)]
        return p, grads, cut(f(2)), cut(f(3).abs()), None, None
    runs = []
    for apart in (False, True):
        p, g, m, v, ms, vs = make(apart)
        masters = None if apart else [p[0], None, p[2], None]
        lb.adamw(p, g, m, v, 3, **HYPER, first_scales=ms, second_scales=vs, masters=masters)
        runs.append([*p, *m, *v, *(ms or []), *(vs or [])])
    for a, b in zip(*runs):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    p, g, m, v, ms, vs = make(False)
    before = [t.clone() for t in (*p, *m, *v)]
    held = torch.zeros(6000, device="cuda")
    for bad in (dict(params=[held[:256], held[255:555], *p[2:]]), dict(grads=[p[0], *g[1:]]), dict(grads=[p[3][1:257], *g[1:]]), dict(first=v),
                dict(params=[*p[:3], held[:5000]], masters=[None, None, None, held[1000:]])):
        with pytest.raises(lb.LibraError):
            lb.adamw(**{**dict(params=p, grads=g, first=m, second=v, step=3, first_scales=ms, second_scales=vs), **bad})
    for t, b in zip((*p, *m, *v), before):
        assert torch.equal(t.view(torch.uint8), b.view(torch.uint8))
