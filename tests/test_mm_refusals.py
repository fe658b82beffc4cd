"""The products of a rank's layer refuse what they cannot do, before touching a device (no GPU needed)."""

import ctypes as C
import types

import pytest
import torch

P16 = 0x1000  # (an aligned address that nothing reads)


def refused(fsb, rc):
    assert rc == fsb.FS_EINVAL and fsb.fs_last_error()


def good(fsb, type_=0):
    """Sizes 3 x 20 x 10, rows of 32, each operand at an address of its own."""
    at = iter(range(P16, 1 << 20, P16))

    def rows(codes):
        return fsb.fs_mm_rows(next(at), 32, P16 if codes else None)

    head = dict(rows=3, in_=20, out=10, type=type_, activation=0)
    e = type_ == 2
    linear = fsb.fs_mm_linear(**head, out_type=0, x=rows(e), w=rows(e), residual=rows(0), y=rows(0), bias=1 << 20)
    gated = fsb.fs_mm_gated(**head, out_type=0, x=rows(e), w_gate=rows(e), w_up=rows(e), y=rows(0))
    grad = fsb.fs_mm_gated_grad(**head, x=rows(0), w_gate=rows(0), w_up=rows(0), dy=rows(0), dx=rows(0), dw_gate=rows(0), dw_up=rows(0))
    return {"fs_linear": linear, "fs_gated_ff": gated, "fs_gated_ff_backward": grad}


def call(fsb, name, args, ws=P16, n=1 << 40):
    return getattr(fsb.lib(), name)(C.byref(args) if args is not None else None, ws, n, None)


CALLS = ["fs_linear", "fs_gated_ff", "fs_gated_ff_backward"]
ROWS = [("fs_linear", r) for r in ("x", "w", "residual", "y")] + [("fs_gated_ff", r) for r in ("x", "w_gate", "w_up", "y")] + [
    ("fs_gated_ff_backward", r) for r in ("x", "w_gate", "w_up", "dy", "dx", "dw_gate", "dw_up")]


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("field,value", [("rows", -1), ("rows", (1 << 24) + 1), ("in_", 0), ("in_", -4), ("in_", (1 << 24) + 1), ("out", -1),
                                         ("out", (1 << 24) + 1), ("type", 3), ("type", -1), ("activation", 5), ("activation", -1)])
def test_heads(fsb, name, field, value):
    a = good(fsb)[name]
    setattr(a, field, value)
    refused(fsb, call(fsb, name, a))


@pytest.mark.parametrize("name", CALLS[:2])
def test_types_that_do_not_go_together(fsb, name):
    for type_, out in ((0, 1), (1, 0), (2, 2), (0, 2), (2, -1)):
        a = good(fsb, type_)[name]
        a.out_type = out
        refused(fsb, call(fsb, name, a))
    refused(fsb, call(fsb, "fs_gated_ff_backward", good(fsb, 2)["fs_gated_ff_backward"]))


@pytest.mark.parametrize("name,rows", ROWS)
@pytest.mark.parametrize("field,value", [("data", P16 + 8), ("data", None), ("stride", 20), ("stride", 8), ("stride", -32), ("stride", 0),
                                         ("stride", 1 << 40), ("scale", P16)])
def test_rows(fsb, name, rows, field, value):
    if rows == "residual" and (field, value) in (("data", None), ("stride", 0)):
        return  # none, and the same row for all
    a = good(fsb)[name]
    setattr(getattr(a, rows), field, value)
    refused(fsb, call(fsb, name, a))


@pytest.mark.parametrize("name,rows", [r for r in ROWS if r[1] in ("x", "w", "w_gate", "w_up") and r[0] != "fs_gated_ff_backward"])
@pytest.mark.parametrize("field,value", [("stride", 24), ("scale", None), ("scale", P16 + 4)])
def test_codes(fsb, name, rows, field, value):
    a = good(fsb, 2)[name]
    setattr(getattr(a, rows), field, value)
    refused(fsb, call(fsb, name, a))


def test_workspace_bias_and_null_structs(fsb):
    for name in CALLS:
        for ws, n in ((None, 1 << 40), (P16 + 16, 1 << 40), (P16, 128)):
            refused(fsb, call(fsb, name, good(fsb)[name], ws, n))
        refused(fsb, call(fsb, name, None))
    need = C.c_int64()
    fsb.lib().fs_mm_workspace_bytes(3, 20, 10, 1, C.byref(need))
    refused(fsb, call(fsb, "fs_gated_ff_backward", good(fsb)["fs_gated_ff_backward"], n=need.value - 1))
    a = good(fsb)["fs_linear"]
    a.bias = P16 + 2
    refused(fsb, call(fsb, "fs_linear", a))
    L = fsb.lib()
    refused(fsb, L.fs_mm_check(None, None))
    refused(fsb, L.fs_mm_check(P16 + 8, None))
    for sizes in ((-1, 1, 1, 0), (1, 0, 1, 0), (1, 1, -1, 0), (1, 1, 1, 2)):
        refused(fsb, L.fs_mm_workspace_bytes(*sizes, C.byref(need)))
    refused(fsb, L.fs_mm_workspace_bytes(1, 1, 1, 0, None))


OUTPUTS = [("fs_linear", "y", ("x", "w")), ("fs_gated_ff", "y", ("x", "w_gate", "w_up"))] + [
    ("fs_gated_ff_backward", o, ("x", "w_gate", "w_up", "dy") + tuple(p for p in ("dx", "dw_gate", "dw_up") if p != o)) for o in ("dx", "dw_gate", "dw_up")]


@pytest.mark.parametrize("name,out,others", OUTPUTS)
def test_outputs_that_overlap(fsb, name, out, others):
    """The same place; the same columns of later rows; columns that meet; a row's end inside another's."""
    for other in others:
        for off in (0, 64, 16, -16, 2 * 64 + 16):
            a = good(fsb)[name]
            getattr(a, out).data = getattr(a, other).data + off
            refused(fsb, call(fsb, name, a))
            assert b"overlap" in fsb.lib().fs_last_error()


def test_residual_and_bias_that_overlap(fsb):
    for off in (64, 16, -16):
        a = good(fsb)["fs_linear"]
        a.residual.data = a.y.data + off
        refused(fsb, call(fsb, "fs_linear", a))
    a = good(fsb)["fs_linear"]
    a.residual.data, a.residual.stride = a.y.data, 0  # one of y's rows for all
    refused(fsb, call(fsb, "fs_linear", a))
    a = good(fsb)["fs_linear"]
    a.bias = a.y.data + 64
    refused(fsb, call(fsb, "fs_linear", a))
    x = fsb.fs_mm_rows(P16, 32, None)
    for off, stride in ((0, 64), (0, 32), (64, 64), (16, 64), (-16, 64)):
        c = fsb.fs_mm_rows(P16 + off, stride, None)
        refused(fsb, fsb.lib().fs_quantise_rows(3, 20, 0, C.byref(x), C.byref(c), 1 << 20, None))


def test_the_workspace_grows_with_every_size(fsb):
    def need(*sizes):
        n = C.c_int64()
        assert fsb.lib().fs_mm_workspace_bytes(*sizes, C.byref(n)) == fsb.FS_OK
        return n.value

    for back in (0, 1):
        for sizes in ((1, 1, 1), (7, 100, 63), (64, 8192, 1280), (4096, 4096, 7168)):
            for i in range(3):
                more = [s + (9 if i == j else 0) for j, s in enumerate(sizes)]
                assert need(*more, back) >= need(*sizes, back) > 0
    assert need(0, 1, 0, 0) > 0


def test_quantise(fsb):
    L = fsb.lib()
    x, c = fsb.fs_mm_rows(P16, 32, None), fsb.fs_mm_rows(P16, 32, None)

    def run(rows=3, n=20, type_=0, x=x, c=c, s=P16):
        return L.fs_quantise_rows(rows, n, type_, C.byref(x) if x else None, C.byref(c) if c else None, s, None)

    for bad in (dict(rows=-1), dict(rows=(1 << 24) + 1), dict(n=0), dict(type_=2), dict(type_=-1), dict(x=None), dict(c=None), dict(s=None),
                dict(s=P16 + 4), dict(x=fsb.fs_mm_rows(P16, 12, None)), dict(c=fsb.fs_mm_rows(P16, 24, None)),
                dict(c=fsb.fs_mm_rows(P16 + 8, 32, None)), dict(x=fsb.fs_mm_rows(None, 32, None))):
        refused(fsb, run(**bad))
    assert run(rows=0) == fsb.FS_OK


def test_calls_without_rows_do_nothing(fsb):
    for name in CALLS[:2]:
        for field in ("rows", "out"):
            a = good(fsb)[name]
            setattr(a, field, 0)
            assert call(fsb, name, a) == fsb.FS_OK


class Rows:
    """What the binding asks of a tensor."""

    def __init__(self, shape, dtype=torch.bfloat16, index=0, stride=None):
        self.shape, self.dtype, self.index, self.strides = shape, dtype, index, stride or (64, 1)[-len(shape):]
        self.device = torch.device("cuda", index) if index >= 0 else torch.device("cpu")

    def stride(self):
        return self.strides

    def get_device(self):
        return self.index

    def data_ptr(self):
        return P16

    def dim(self):
        return len(self.shape)

    def element_size(self):
        return self.dtype.itemsize

    def is_floating_point(self):
        return self.dtype.is_floating_point

    def is_contiguous(self):
        return True


@pytest.fixture
def binding(fsb, monkeypatch):
    """The binding with a library that must not be reached, device 0 current."""

    def reached():
        raise AssertionError("the library was called")

    monkeypatch.setattr(fsb, "lib", reached)
    monkeypatch.setattr(fsb, "_current_device", lambda: 0, raising=False)
    monkeypatch.setattr(fsb, "_current_stream", lambda index: 0)
    return fsb


def tensors(**other):
    t = dict(x=Rows((3, 20)), w=Rows((10, 20)), y=Rows((3, 10)), bias=Rows((10,)), residual=Rows((3, 10)), u=Rows((10, 20)), dy=Rows((3, 10)),
             dx=Rows((3, 20)), dw=Rows((10, 20)), dv=Rows((10, 20)), work=types.SimpleNamespace(index=0, address=P16, bytes=1 << 30))
    t.update(other)
    return types.SimpleNamespace(**t)


def calls(fsb, t):
    yield lambda: fsb.fs_linear(t.x, t.w, t.y, bias=t.bias, residual=t.residual, workspace=t.work)
    yield lambda: fsb.fs_gated_ff(t.x, t.w, t.u, t.y, workspace=t.work)
    yield lambda: fsb.fs_gated_ff_backward(t.x, t.w, t.u, t.dy, t.dx, t.dw, t.dv, workspace=t.work)


def test_good_tensors_reach_the_library(binding):
    for c in calls(binding, tensors()):
        with pytest.raises(AssertionError, match="the library was called"):
            c()


@pytest.mark.parametrize("which,bad,word", [
    ("x", Rows((3, 21)), "is \\["), ("w", Rows((10, 20), torch.float16), "bfloat16"), ("x", Rows((3, 20), torch.float32), "float32, not"),
    ("x", Rows((3, 20), index=1), "cuda:0"), ("w", Rows((10, 20), index=-1), "cuda:0"), ("x", Rows((3, 20), stride=(1, 3)), "contiguous"),
    ("work", types.SimpleNamespace(index=1, address=P16, bytes=1 << 30), "workspace is on cuda:1")])
def test_tensors_that_every_call_refuses(binding, which, bad, word):
    for c in calls(binding, tensors(**{which: bad})):
        with pytest.raises(ValueError, match=word):
            c()


@pytest.mark.parametrize("at,which,bad", [
    (0, "y", Rows((3, 11))), (0, "y", Rows((4, 10))), (0, "residual", Rows((3, 10), torch.float16)), (0, "bias", Rows((11,))),
    (0, "bias", Rows((10,), index=1)), (0, "bias", Rows((10,), torch.float32)), (1, "u", Rows((11, 20))), (1, "y", Rows((3, 10), torch.float32)),
    (2, "dy", Rows((3, 11))), (2, "dx", Rows((3, 21))), (2, "dw", Rows((11, 20))), (2, "dv", Rows((10, 20), torch.float16))])
def test_tensors_that_one_call_refuses(binding, at, which, bad):
    with pytest.raises(ValueError):
        list(calls(binding, tensors(**{which: bad})))[at]()


def test_scales_activations_and_rows_to_quantise(binding):
    fsb, t = binding, tensors()
    f = Rows((3,), torch.float32)
    for bad in (Rows((4,), torch.float32), Rows((3,), torch.float64), Rows((3,), torch.int32), Rows((3,), torch.float32, 1), Rows((3, 1), torch.float32)):
        with pytest.raises(ValueError, match="scales"):
            fsb.fs_linear(t.x, t.w, t.y, x_scale=bad, workspace=t.work)
    with pytest.raises(ValueError, match="activation"):
        fsb.fs_linear(t.x, t.w, t.y, activation="swish", workspace=t.work)
    c = Rows((3, 20), torch.uint8)
    with pytest.raises(AssertionError, match="the library was called"):
        fsb.fs_quantise_rows(t.x, c, f)
    for x, y, s in ((t.x, Rows((3, 20)), f), (t.x, Rows((3, 21), torch.uint8), f), (t.x, c, Rows((4,), torch.float32)),
                    (Rows((3, 20), torch.float32), c, f), (Rows((3, 20), index=1), c, f), (t.x, Rows((3, 20), torch.uint8, 1), f)):
        with pytest.raises(ValueError):
            fsb.fs_quantise_rows(x, y, s)


def test_scales_that_overlap(fsb):
    for name, scaled in (("fs_linear", ("x", "w")), ("fs_gated_ff", ("x", "w_gate", "w_up"))):
        for rows in scaled:
            for off in (0, 16, 2 * 64 + 16, -16 if rows != "x" else 0):  # (10 rows' scales, or 3: 40 and 12 bytes)
                a = good(fsb, 2)[name]
                getattr(a, rows).scale = a.y.data + off
                refused(fsb, call(fsb, name, a))
                assert b"overlap" in fsb.lib().fs_last_error()
    x, c = fsb.fs_mm_rows(P16, 32, None), fsb.fs_mm_rows(4 * P16, 32, None)
    for scale in (P16, P16 + 32, 4 * P16, 4 * P16 + 64):
        refused(fsb, fsb.lib().fs_quantise_rows(3, 20, 0, C.byref(x), C.byref(c), scale, None))
        assert b"overlap" in fsb.lib().fs_last_error()


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("sizes", [(1 << 20, 1 << 20, 1), (1 << 24, 1, 1 << 16), (1, 1 << 24, 1 << 16)])
def test_operands_beyond_any_memory(fsb, name, sizes):
    a = good(fsb)[name]
    a.rows, a.in_, a.out = sizes
    refused(fsb, call(fsb, name, a, n=1 << 62))
    assert b"2^40" in fsb.lib().fs_last_error()
