"""What the calls at the ends of a training step refuse, through the C ABI (arguments are looked at before anything touches a GPU) and
through the binding."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2506_22714_amd import binding as lb

OK, E = lb.OK, lb.ERR
BUF = np.zeros(4096, dtype=np.uint8)
AT = -(-BUF.ctypes.data // 256) * 256           # never read or written: every call here is refused, or has nothing to do


def embedding(**kw):
    a = dict(table=AT, rows=4, width=8, ld_table=8, dtype=lb.F16, index=AT, index_type=lb.INDEX_I64, n=2, scale=1.0, out=AT, ld_out=8)
    a.update(kw)
    return lb.lib().libra_embedding(*a.values(), None)


def scatter(**kw):
    a = dict(dout=AT, ld_dout=8, dtype=lb.F16, index=AT, index_type=lb.INDEX_I64, n=2, rows=4, width=8, scale=1.0, out=AT, ld_out=8, ws=AT, ws_bytes=1 << 30)
    a.update(kw)
    return lb.lib().libra_embedding_backward(*a.values(), None)


def log_probs(**kw):
    a = dict(logits=AT, n=2, classes=8, ld=8, dtype=lb.F32, targets=AT, index_type=lb.INDEX_I64, top=2, scale=1.0, target_out=AT, entropy=AT,
             top_out=AT, top_index=AT, stats=AT, ws=AT, ws_bytes=1 << 30)
    a.update(kw)
    return lb.lib().libra_log_probs(*a.values(), None)


def log_probs_backward(**kw):
    a = dict(logits=AT, n=2, classes=8, ld=8, dtype=lb.F32, targets=AT, index_type=lb.INDEX_I64, top=2, scale=1.0, entropy=AT, stats=AT,
             top_index=AT, d_target=AT, d_entropy=AT, d_top=AT, out=AT, ld_out=8)
    a.update(kw)
    return lb.lib().libra_log_probs_backward(*a.values(), None)


def adamw(bits=32, tensors=None, count=None, opts=True, **kw):
    o = lb.AdamwOpts(state_bits=bits, lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.0, step=1)
    t = dict(param=AT, grad=AT, first=AT, second=AT, first_scales=AT, second_scales=AT, n=4, dtype=lb.F32)
    for k, v in kw.items():
        if k in t or k in ("master", "number"):
            t[k] = v
        else:
            setattr(o, k, v)
    table = (lb.AdamwTensor * 1)(lb.AdamwTensor(**t)) if tensors is None else tensors
    return lb.lib().libra_adamw(table, 1 if count is None else count, C.byref(o) if opts else None, None)


@pytest.mark.parametrize("want,kw", [
    ("SHAPE", dict(n=-1)), ("SHAPE", dict(rows=-1)), ("SHAPE", dict(width=0)), ("SHAPE", dict(ld_table=7)), ("SHAPE", dict(ld_out=7)),
    ("DTYPE", dict(dtype=3)), ("OPTION", dict(index_type=2)), ("NULL", dict(table=None)), ("NULL", dict(index=None)), ("NULL", dict(out=None)),
    ("BUFFER", dict(table=AT + 1)), ("BUFFER", dict(index=AT + 4)), ("BUFFER", dict(out=AT + 1)), ("BUFFER", dict(dtype=lb.F32, out=AT + 2)),
])
def test_embedding_refuses(want, kw):
    assert embedding(**kw) == E[want]


@pytest.mark.parametrize("want,kw", [
    ("SHAPE", dict(n=-1)), ("SHAPE", dict(rows=-1)), ("SHAPE", dict(width=0)), ("SHAPE", dict(ld_dout=7)), ("SHAPE", dict(ld_out=7)),
    ("TOO_LARGE", dict(n=1 << 31)), ("TOO_LARGE", dict(rows=(1 << 31) - 1)), ("UNSUPPORTED", dict(width=(1 << 21) + 1, ld_dout=1 << 22, ld_out=1 << 22)), ("DTYPE", dict(dtype=-1)), ("OPTION", dict(index_type=-1)),
    ("NULL", dict(dout=None)), ("NULL", dict(index=None)), ("NULL", dict(out=None)), ("NULL", dict(n=100000, ws=None)),
    ("BUFFER", dict(n=100000, ws=AT + 128)), ("BUFFER", dict(n=100000, ws_bytes=8)), ("BUFFER", dict(dout=AT + 1)), ("BUFFER", dict(index=AT + 4)), ("BUFFER", dict(out=AT + 1)),
])
def test_embedding_backward_refuses(want, kw):
    assert scatter(**kw) == E[want]


@pytest.mark.parametrize("want,kw", [
    ("SHAPE", dict(n=-1)), ("SHAPE", dict(classes=0, ld=0, top=0)), ("SHAPE", dict(ld=7)), ("SHAPE", dict(top=-1)), ("SHAPE", dict(top=9)),
    ("TOO_LARGE", dict(n=1 << 31)), ("TOO_LARGE", dict(classes=1 << 31, ld=1 << 31)), ("UNSUPPORTED", dict(classes=100, ld=100, top=65)),
    ("DTYPE", dict(dtype=3)), ("OPTION", dict(index_type=2)), ("OPTION", dict(scale=0.0)), ("OPTION", dict(scale=-1.0)),
    ("OPTION", dict(scale=float("inf"))), ("OPTION", dict(scale=float("nan"))), ("NULL", dict(logits=None)), ("BUFFER", dict(logits=AT + 2)),
    ("BUFFER", dict(targets=AT + 4)), ("NULL", dict(entropy=None)), ("NULL", dict(stats=None)), ("NULL", dict(top_index=None)),
    ("BUFFER", dict(top_index=AT + 4)), ("BUFFER", dict(entropy=AT + 2)), ("BUFFER", dict(stats=AT + 2)),
])
def test_log_probs_refuse_both_ways(want, kw):
    assert log_probs(**kw) == E[want]
    assert log_probs_backward(**kw) == E[want]


def test_log_probs_refuse_one_way():
    assert log_probs(target_out=None) == E["NULL"]
    assert log_probs(top_out=None) == E["NULL"]
    assert log_probs(top_out=AT + 2) == E["BUFFER"]
    assert log_probs_backward(ld_out=7) == E["SHAPE"]
    assert log_probs_backward(out=None) == E["NULL"]
    assert log_probs_backward(targets=None) == E["NULL"]            # a gradient of targets that are not there
    for name in ("d_target", "d_entropy", "d_top"):
        assert log_probs_backward(**{name: AT + 2}) == E["BUFFER"]


@pytest.mark.parametrize("want,kw", [
    ("SHAPE", dict(n=-1)), ("SHAPE", dict(count=-1)), ("NULL", dict(opts=False)), ("DTYPE", dict(dtype=3)), ("OPTION", dict(struct_size=4)),
    ("OPTION", dict(state_bits=16)), ("OPTION", dict(beta1=1.0)), ("OPTION", dict(beta1=-0.1)), ("OPTION", dict(beta2=1.0)), ("OPTION", dict(beta2=float("nan"))),
    ("OPTION", dict(eps=-1.0)), ("OPTION", dict(eps=float("inf"))), ("OPTION", dict(lr=float("nan"))), ("OPTION", dict(weight_decay=float("inf"))),
    ("OPTION", dict(step=0)), ("BUFFER", dict(step_dev=AT + 4)), ("BUFFER", dict(lr_dev=AT + 2)), ("TOO_LARGE", dict(n=1 << 60)),
    ("NULL", dict(param=None)), ("NULL", dict(grad=None)), ("NULL", dict(first=None)), ("NULL", dict(second=None)),
    ("NULL", dict(bits=8, first_scales=None)), ("NULL", dict(bits=8, second_scales=None)), ("BUFFER", dict(param=AT + 2)), ("BUFFER", dict(grad=AT + 1)),
    ("BUFFER", dict(first=AT + 2)), ("BUFFER", dict(second=AT + 1)), ("BUFFER", dict(master=AT + 2)), ("BUFFER", dict(bits=8, first_scales=AT + 2)),
])
def test_adamw_refuses(want, kw):
    assert adamw(**kw) == E[want]


def test_nothing_to_do_is_no_error():
    assert embedding(n=0, table=None, index=None, out=None) == OK
    assert scatter(rows=0, dout=None, index=None, out=None, ws=None) == OK
    assert log_probs(n=0, logits=None, targets=None, target_out=None, entropy=None, top_out=None, top_index=None, stats=None) == OK
    assert log_probs_backward(n=0, logits=None, out=None) == OK
    assert adamw(count=0) == OK
    assert adamw(n=0, param=None, grad=None, first=None, second=None) == OK
    n = C.c_size_t()
    assert lb.lib().libra_embedding_backward_workspace(5, 1 << 31, 4, C.byref(n)) == E["TOO_LARGE"]
    assert lb.lib().libra_embedding_backward_workspace(5, 10, 4, None) == E["NULL"]
    assert lb.lib().libra_log_probs_workspace(5, 10, 11, C.byref(n)) == E["SHAPE"]
    assert lb.lib().libra_log_probs_workspace(5, 10, 4, None) == E["NULL"]


def test_the_binding_wants_gpu_tensors_of_the_right_kind():
    table, ids = torch.zeros(4, 8), torch.zeros(3, dtype=torch.int64)
    for call in (lambda: lb.embedding(table, ids), lambda: lb.embedding(table.double(), ids), lambda: lb.embedding(table[0], ids),
                 lambda: lb.embedding(table.t(), ids), lambda: lb.embedding([1.0], ids), lambda: lb.embedding_backward(table, ids, 5),
                 lambda: lb.log_probs(table), lambda: lb.log_probs(table.int()), lambda: lb.log_probs_backward(table, None)):
        with pytest.raises(ValueError):
            call()
    p = [torch.zeros(4)]
    for call in (lambda: lb.adamw(p, p, p, p, 1), lambda: lb.adamw(p, [], p, p, 1), lambda: lb.adamw(p, p, p, p, 1, first_scales=p),
                 lambda: lb.adamw(p, p, p, p, 1, masters=[])):
        with pytest.raises(ValueError):
            call()
    lb.adamw([], [], [], [], 1)


def test_the_optimizer_refuses():
    from paper_2506_22714_amd.optim import AdamW
    p = [torch.nn.Parameter(torch.zeros(4))]
    for kw in (dict(state_bits=16), dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(eps=-1.0), dict(lr=torch.tensor(1e-3))):
        with pytest.raises(ValueError):
            AdamW(p, **kw)


def test_widths_that_32_bits_do_not_hold():
    """(Tensors without rows: they take no memory.)"""
    for width in (0, 1 << 31, (1 << 32) + 8):
        with pytest.raises(ValueError, match="elements"):
            lb._width(torch.empty(0, width), "table")
    assert lb._width(torch.empty(0, (1 << 31) - 1), "table") == (1 << 31) - 1


def test_adamw_refuses_arrays_that_overlap():
    """Addresses that nothing is read from: the call is refused before."""
    def call(bits, dtype=lb.F32, n=300, tensors=2, **places):
        table = (lb.AdamwTensor * tensors)()
        for k in range(tensors):
            at = dict(zip(("param", "grad", "first", "second", "first_scales", "second_scales", "master"), range((1 + 7 * k) << 20, (8 + 7 * k) << 20, 1 << 20)))
            table[k] = lb.AdamwTensor(**at, n=n, dtype=dtype)
        for name, value in places.items():
            setattr(table[tensors - 1], name, value)
        return adamw(bits, tensors=table, count=tensors)
    size = {"param": 1200, "first": 1200, "second": 1200, "master": 1200, "first_scales": 8, "second_scales": 8, "grad": 1200}
    first = {name: (k + 1) << 20 for k, name in enumerate(("param", "grad", "first", "second", "first_scales", "second_scales", "master"))}
    for bits in (32, 8):
        for tensors in (2, 40):
            for name in size:
                for other, begin in first.items():
                    if bits == 32 and "scales" in name + other or name == other == "grad":
                        continue
                    bytes_of = lambda x: 300 if bits == 8 and x in ("first", "second") else size[x]       # noqa: E731
                    for at in (begin, begin + bytes_of(other) - 4, begin - bytes_of(name) + 4):
                        assert call(bits, tensors=tensors, **{name: at}) == E["BUFFER"], (bits, tensors, name, other)


def test_a_row_beside_the_columns_that_are_written():
    """By places: a result lies on its input or not, whichever of them has a single row."""
    held = torch.zeros(12, 16)
    places = torch.arange(12 * 16).view(12, 16)
    def cut(x, rows, cols):
        return x[slice(*rows), slice(*cols)]
    some = [((a, b), (c, d)) for a, b in ((0, 12), (0, 1), (5, 6), (11, 12), (3, 7)) for c, d in ((0, 16), (0, 8), (8, 16), (3, 9), (8, 12), (15, 16))]
    apart = 0
    for one in some:
        for two in some:
            out, t = cut(held, *one), cut(held, *two)
            lie_on = bool(torch.isin(cut(places, *one).contiguous(), cut(places, *two).contiguous()).any())
            if lie_on:
                with pytest.raises(ValueError, match="overlaps"):
                    lb._apart(out, t, "t")
            else:
                lb._apart(out, t, "t")
                apart += 1
    assert apart > 300
    with pytest.raises(ValueError, match="overlaps"):
        lb._apart(held.view(24, 8)[1:3], held[:, :8], "t")          # rows of other distances: not looked at any further


def test_the_largest_scale():
    for scale in (1.8e38, 3e38):
        assert log_probs(scale=scale) == E["OPTION"] and log_probs_backward(scale=scale) == E["OPTION"]
    assert log_probs(scale=2.0 ** 127, n=0) == OK


def test_a_checkpoint_of_a_group_without_parameters():
    from paper_2506_22714_amd.optim import AdamW
    make = lambda lr: AdamW([{"params": [torch.nn.Parameter(torch.zeros(4))]}, {"params": [], "lr": lr}])      # noqa: E731
    again = make(0.5)
    again.load_state_dict(make(0.25).state_dict())
    assert [g["lr"] for g in again.param_groups] == [1e-3, 0.25]
    rate = torch.full((1,), 0.125)
    make_tensor = lambda lr: AdamW([{"params": [torch.nn.Parameter(torch.zeros(4))]}, {"params": [], "lr": lr}], capturable=True)      # noqa: E731
    again = make_tensor(torch.zeros(1))
    again.load_state_dict(make_tensor(rate).state_dict())
    assert float(again.param_groups[1]["lr"]) == 0.125


@pytest.mark.parametrize("capturable", [False, True])
def test_a_step_of_a_group_without_parameters(capturable, monkeypatch):
    """It has no GPU to count on."""
    monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: False)
    from paper_2506_22714_amd.optim import AdamW
    opt = AdamW([{"params": []}, {"params": [torch.nn.Parameter(torch.zeros(4))]}], capturable=capturable)
    for _ in range(2):
        opt.step()                      # no parameter has a gradient
    if capturable:
        assert int(opt.param_groups[1]["step"]) == 2 and "step" not in opt.param_groups[0]
