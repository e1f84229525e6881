"""The operators between the layers: sizes, what they refuse before any device work, and their oracle (no GPU needed)."""
import ctypes as C

import numpy as np
import pytest
import torch

from between_util import e4m3, in_8_bits, kept, numbers, philox
from paper_2006_02924_amd import binding as B

FAR = 1 << 40      # addresses that are never used


def form(**kw):
    f = B.JoinForm()
    f.struct_bytes, f.dtype, f.stream_dtype, f.norm, f.after, f.before, f.width = C.sizeof(B.JoinForm), B.F32, B.F32, 0, 1, 1, 40
    f.eps, f.residual_scale, f.dropout, f.seed = 1e-5, 1.0, 0.1, 7
    f.after_weight, f.after_bias, f.gate, f.before_weight, f.before_bias = 0, 40, 80, 120, 160
    for k, v in kw.items():
        setattr(f, k, v)
    return f


FORM = {name for name, _ in B.JoinForm._fields_}


def split_form(kw):
    return form(**{k: v for k, v in kw.items() if k in FORM}), {k: v for k, v in kw.items() if k not in FORM}


def dropout(lib, x=FAR, dtype=B.F32, stride=40, rows=4, width=40, p=0.1, seed=1, step=5 * FAR, out=2 * FAR, out_stride=40):
    return lib.adasum_dropout(x, dtype, stride, rows, width, p, seed, step, out, out_stride, None)


def join(lib, **kw):
    f, kw = split_form(kw)
    a = dict(params=FAR, param_dtype=B.F32, step=8 * FAR, x=2 * FAR, x_stride=40, residual=3 * FAR, residual_stride=40, rows=4, h=4 * FAR, h_stride=40,
             y=5 * FAR, y_stride=40)
    a.update(kw)
    return lib.adasum_join(C.byref(f), *a.values(), None)


def join_grad(lib, **kw):
    f, kw = split_form(kw)
    a = dict(params=FAR, param_dtype=B.F32, step=8 * FAR, x=2 * FAR, x_stride=40, h=3 * FAR, h_stride=40, dy=4 * FAR, dy_stride=40, dh=5 * FAR, dh_stride=40,
             rows=4, dx=6 * FAR, dx_stride=40, dresidual=7 * FAR, dresidual_stride=40, grad=9 * FAR, grad_dtype=B.F32, accumulate=0, ws=10 * FAR,
             ws_bytes=1 << 30)
    a.update(kw)
    return lib.adasum_join_grad(C.byref(f), *a.values(), None)


def store8(lib, params=FAR, dtype=B.F32, offset=0, outputs=16, width=40, weight=2 * FAR):
    return lib.adasum_linear_store(params, dtype, offset, outputs, width, weight, None)


def linear(lib, weight=FAR, outputs=16, width=40, x=2 * FAR, dtype=B.F32, x_stride=40, rows=4, params=3 * FAR, param_dtype=B.F32, bias=0, out=4 * FAR,
            out_dtype=B.F32, out_stride=16, ws=5 * FAR, ws_bytes=1 << 30):
    return lib.adasum_linear(weight, outputs, width, x, dtype, x_stride, rows, params, param_dtype, bias, out, out_dtype, out_stride, ws, ws_bytes, None)


def linear_grad(lib, weight=FAR, outputs=16, width=40, dy=2 * FAR, dtype=B.F32, dy_stride=16, rows=4, dx=4 * FAR, dx_dtype=B.F32, dx_stride=40,
                 ws=5 * FAR, ws_bytes=1 << 30):
    return lib.adasum_linear_grad(weight, outputs, width, dy, dtype, dy_stride, rows, dx, dx_dtype, dx_stride, ws, ws_bytes, None)


NAN = float("nan")


@pytest.mark.parametrize("call, wrong", [
    (dropout, [dict(x=None), dict(out=None), dict(p=-0.1), dict(p=1.1), dict(p=NAN), dict(rows=-1), dict(width=-1), dict(rows=1 << 31),
               dict(width=(1 << 24) + 1), dict(stride=-40), dict(out_stride=39), dict(stride=1 << 50)]),
    (join, [dict(params=None), dict(x=None), dict(h=None, before=0, y=None), dict(y=None), dict(before=0), dict(struct_bytes=8), dict(after=2),
            dict(before=-1), dict(width=-1), dict(eps=0.0), dict(eps=-1.0), dict(eps=NAN), dict(eps=1e-39), dict(eps=1e39), dict(residual_scale=NAN),
            dict(residual_scale=1e39), dict(dropout=1.5), dict(rows=-1), dict(rows=1 << 31), dict(h_stride=39), dict(y_stride=39), dict(x_stride=-1),
            dict(gate=1 << 50)]),
    (join_grad, [dict(params=None), dict(grad=None), dict(x=None), dict(h=None), dict(dy=None), dict(dx=None), dict(dh=None, before=0), dict(accumulate=2),
                 dict(struct_bytes=0), dict(rows=-1), dict(dx_stride=39), dict(dresidual_stride=39), dict(dy_stride=-1), dict(dropout=-1.0)]),
    (store8, [dict(params=None), dict(weight=None), dict(offset=-1), dict(outputs=-1), dict(width=-1), dict(outputs=(1 << 24) + 1), dict(offset=1 << 50),
              dict(outputs=1 << 24, width=1 << 24)]),
    (linear, [dict(weight=None), dict(x=None), dict(out=None), dict(params=None), dict(outputs=-1), dict(width=-1), dict(rows=-1), dict(rows=1 << 31),
               dict(out_stride=15), dict(x_stride=-1), dict(width=(1 << 24) + 1)]),
    (linear_grad, [dict(weight=None), dict(dy=None), dict(dx=None), dict(rows=-1), dict(dx_stride=39), dict(outputs=(1 << 24) + 1)]),
])
def test_invalid_arguments(lib, call, wrong):
    for kw in wrong:
        assert call(lib, **kw) == B.ERR_INVALID_ARG, kw


@pytest.mark.parametrize("call, wrong", [
    (dropout, [dict(dtype=B.F64), dict(dtype=9)]),
    (join, [dict(dtype=B.F64), dict(stream_dtype=B.BF16), dict(dtype=B.BF16, stream_dtype=B.F16), dict(stream_dtype=B.F64), dict(norm=2), dict(width=8193),
            dict(param_dtype=B.F64)]),
    (join_grad, [dict(dtype=B.F64), dict(norm=-1), dict(width=8193), dict(param_dtype=B.F64), dict(grad_dtype=B.F64)]),
    (store8, [dict(dtype=B.F64), dict(dtype=-1)]),
    (linear, [dict(dtype=B.F64), dict(out_dtype=B.F64), dict(param_dtype=B.F64)]),
    (linear_grad, [dict(dtype=4), dict(dx_dtype=B.F64)]),
])
def test_unsupported(lib, call, wrong):
    for kw in wrong:
        assert call(lib, **kw) == B.ERR_UNSUPPORTED, kw


@pytest.mark.parametrize("call, names", [(dropout, ("x", "out")), (join, ("params", "x", "residual", "h", "y")),
                                         (join_grad, ("params", "x", "h", "dy", "dh", "dx", "dresidual", "grad")), (store8, ("params", "weight")),
                                         (linear, ("weight", "x", "params", "out")), (linear_grad, ("weight", "dy", "dx"))])
def test_misaligned_pointers(lib, call, names):
    for name in names:
        assert call(lib, **{name: 99 * FAR + 8}) == B.ERR_MISALIGNED, name
    if call in (dropout, join, join_grad):
        assert call(lib, step=99 * FAR + 4) == B.ERR_MISALIGNED


def test_results_may_not_overlap(lib):
    assert dropout(lib, out=FAR + 16) == dropout(lib, out=FAR, out_stride=48) == dropout(lib, step=2 * FAR + 8) == B.ERR_ALIAS
    assert join(lib, h=2 * FAR) == join(lib, y=2 * FAR) == join(lib, y=3 * FAR) == join(lib, y=4 * FAR + 16) == B.ERR_ALIAS
    assert join(lib, h=3 * FAR, h_stride=48) == join(lib, y=FAR + 640) == join(lib, h=FAR + 16) == join(lib, step=4 * FAR) == B.ERR_ALIAS
    for name, at in (("dx", 2), ("dx", 3), ("dx", 4), ("dx", 5), ("dx", 7), ("dx", 9), ("dresidual", 3), ("dresidual", 9), ("grad", 1), ("grad", 4), ("ws", 2),
                     ("ws", 6), ("ws", 9), ("ws", 1), ("dx", 8)):
        assert join_grad(lib, **{name: at * FAR}) == B.ERR_ALIAS, (name, at)
    assert join_grad(lib, dresidual=5 * FAR, dresidual_stride=48) == B.ERR_ALIAS           # dh itself, with other rows
    assert join_grad(lib, gate=119) == join_grad(lib, gate=0) == B.ERR_ALIAS               # the gate's gradient and another vector's
    assert store8(lib, weight=FAR + 16) == B.ERR_ALIAS
    assert linear(lib, out=FAR) == linear(lib, out=2 * FAR) == linear(lib, out=3 * FAR) == B.ERR_ALIAS
    assert linear_grad(lib, dx=FAR + 1024) == linear_grad(lib, dx=2 * FAR) == B.ERR_ALIAS


def test_workspaces(lib):
    n = C.c_size_t(0)
    assert lib.adasum_join_grad_workspace_bytes(C.byref(form()), 4, C.byref(n)) == B.OK and n.value > 0
    assert join_grad(lib, ws_bytes=n.value - 1) == join_grad(lib, ws=None) == join_grad(lib, ws=10 * FAR + 16) == B.ERR_WORKSPACE
    none = form(after_weight=-1, after_bias=-1, gate=-1, before_weight=-1, before_bias=-1)
    assert lib.adasum_join_grad_workspace_bytes(C.byref(none), 4, C.byref(n)) == B.OK and n.value == 0
    assert lib.adasum_join_grad_workspace_bytes(C.byref(form(width=9000)), 4, C.byref(n)) == B.ERR_UNSUPPORTED
    assert lib.adasum_join_grad_workspace_bytes(C.byref(form()), -4, C.byref(n)) == B.ERR_INVALID_ARG
    assert lib.adasum_join_grad_workspace_bytes(C.byref(form()), 4, None) == B.ERR_INVALID_ARG
    assert lib.adasum_join_grad_workspace_bytes(None, 4, C.byref(n)) == B.ERR_INVALID_ARG
    assert lib.adasum_linear_workspace_bytes(4096, 1024, 1024, B.BF16, C.byref(n)) == B.OK
    if n.value:
        big = dict(rows=4096, outputs=1024, width=1024, out_dtype=B.BF16, x_stride=1024, out_stride=1024)
        assert linear(lib, ws_bytes=n.value - 1, **big) == linear(lib, ws=None, **big) == B.ERR_WORKSPACE
        assert linear(lib, ws=2 * FAR, **big) == linear(lib, ws=4 * FAR, **big) == linear(lib, ws=FAR, **big) == linear(lib, ws=3 * FAR, **big) == B.ERR_ALIAS
    assert lib.adasum_linear_workspace_bytes(4, 40, 16, B.F64, C.byref(n)) == B.ERR_UNSUPPORTED
    assert lib.adasum_linear_workspace_bytes(-4, 40, 16, B.F32, C.byref(n)) == B.ERR_INVALID_ARG
    assert lib.adasum_linear_workspace_bytes(4, 40, 16, B.F32, None) == B.ERR_INVALID_ARG


@pytest.mark.parametrize("outputs, width, want", [(0, 5, 0), (5, 0, 0), (1, 1, 128 + 128 + 16), (128, 128, 2 * 128 * 128 + 16), (129, 300, 129 * 384 + 300 * 256 + 16)])
def test_weight_bytes(lib, outputs, width, want):
    n = C.c_size_t(1)
    assert lib.adasum_linear_bytes(outputs, width, C.byref(n)) == B.OK and n.value == want
    assert lib.adasum_linear_bytes(-1, width, C.byref(n)) == B.ERR_INVALID_ARG
    assert lib.adasum_linear_bytes(outputs, width, None) == B.ERR_INVALID_ARG


def test_nothing_to_do_needs_no_device(lib):
    assert dropout(lib, rows=0, x=None, out=None) == dropout(lib, width=0, x=None, out=None) == B.OK
    assert join(lib, rows=0, x=None, residual=None, h=None, y=None) == B.OK
    assert join_grad(lib, width=0) == B.OK
    assert store8(lib, outputs=0, params=None, weight=None) == store8(lib, width=0, params=None, weight=None) == B.OK
    assert linear(lib, rows=0, x=None, out=None, ws=None) == linear(lib, outputs=0, weight=None, out=None, params=None) == B.OK
    assert linear_grad(lib, width=0, weight=None, dx=None) == B.OK


def test_binding_refuses():
    x = torch.zeros(4, 40)
    for call in (lambda: B.adasum_dropout(x, 0.1, 1), lambda: B.Join(40, torch.float32, norm="batch"), lambda: B.Join(40, torch.float32, gate=-3),
                 lambda: B.adasum_join(B.Join(40, torch.float32), None, x), lambda: B.adasum_join(B.Join(40, torch.float32, gate=0), None, x),
                 lambda: B.adasum_join(B.Join(40, torch.float16), None, x), lambda: B.adasum_join(B.Join(41, torch.float32), None, x),
                 lambda: B.adasum_join_grad(B.Join(40, torch.float32), None, None, dy=x),
                 lambda: B.adasum_join_grad(B.Join(40, torch.float32, before=False), None, None),
                 lambda: B.adasum_join_grad(B.Join(40, torch.float32, gate=0), x, x, h=x, dy=x),
                 lambda: B.Weight8(4, 40, data=torch.zeros(9, dtype=torch.uint8)), lambda: B.adasum_linear_store(x.view(-1), 0, 4, 40),
                 lambda: B.adasum_linear_store(x.view(-1), 1, 4, 40), lambda: B.adasum_linear(B.Weight8(4, 40, device="cpu"), x),
                 lambda: B.adasum_linear(B.Weight8(4, 41, device="cpu"), x), lambda: B.adasum_linear_grad(B.Weight8(40, 4, device="cpu"), x)):
        with pytest.raises(ValueError):
            call()


# ---- the oracle --------------------------------------------------------------------------

@pytest.mark.parametrize("counter, key, want", [
    # known answers that the method's authors publish
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
])
def test_known_answers_of_the_generator(counter, key, want):
    assert tuple(int(w) for w in philox(counter, key)) == want


def test_the_mask_is_fair():
    n, width = 400, 1000
    for p in (0.0, 0.1, 0.5, 1.0):
        keep, factor = kept(n, width, p, 12345 + (77 << 40), 3)
        # the share that is kept, within five deviations of n * width draws; its expected product with the factor is one
        assert abs(keep.mean() - (1 - p)) <= 5 * np.sqrt(p * (1 - p) / (n * width)) + 2 ** -17
        assert p == 1.0 or abs(factor * (1 - np.floor(65536 * p + 0.5) / 65536) - 1) < 1e-15
    assert not np.array_equal(numbers(3, 9, 1, 0), numbers(3, 9, 1, 1)) and not np.array_equal(numbers(3, 9, 1, 0), numbers(3, 9, 1 << 32, 0))
    assert not np.array_equal(numbers(3, 9, 1, 0), numbers(3, 9, 1, 1 << 32))


def test_8_bit_numbers():
    # every e4m3 number stays what it is, and the middle between two goes to the even one
    bits = torch.arange(0, 127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert bits[-1] == 448 and np.array_equal(e4m3(bits), bits) and np.array_equal(e4m3(-bits), -bits)
    mid = (bits[1:] + bits[:-1]) / 2
    even = np.where(np.arange(126) % 2 == 0, bits[:-1], bits[1:])
    assert np.array_equal(e4m3(mid), even)
    v, e = in_8_bits(np.array([[448.0, 1.0], [448.1, 1.0], [0.0, 0.0], [np.inf, 2.0]]), 1)
    assert e[:, 0].tolist() == [0, 1, -120, -7] and v[0].tolist() == [448.0, 1.0] and v[1].tolist() == [448.0, 1.0] and np.isnan(v[3, 0]) and v[3, 1] == 2.0
