"""The operators that fill a worker's gradient buffer: sizes, and what they refuse before any device work (no GPU needed)."""
import ctypes as C

import pytest

from paper_2006_02924_amd import binding as B

FAR = 1 << 40      # addresses that are never used


def embedding(lib, params=FAR, dtype=B.F32, offset=0, rows=10, width=8, ids=2 * FAR, id_type=B.ID_I64, n=4, out=3 * FAR, out_dtype=B.F32,
              stride=8):
    return lib.adasum_embedding(params, dtype, offset, rows, width, ids, id_type, n, 1.0, out, out_dtype, stride, None)


def embedding_grad(lib, dy=FAR, dtype=B.F32, stride=8, ids=2 * FAR, id_type=B.ID_I64, n=4, grad=3 * FAR, grad_dtype=B.F32, offset=0, rows=10,
                   width=8, accumulate=0, ws=4 * FAR, ws_bytes=1 << 30):
    return lib.adasum_embedding_grad(dy, dtype, stride, ids, id_type, n, 1.0, grad, grad_dtype, offset, rows, width, accumulate, ws, ws_bytes,
                                     None)


def store(lib, x=FAR, dtype=B.F32, stride=40, rows=4, width=40, kept=2 * FAR):
    return lib.adasum_checkpoint_store(x, dtype, stride, rows, width, kept, None)


def load(lib, kept=FAR, rows=4, width=40, out=2 * FAR, dtype=B.F32, stride=40):
    return lib.adasum_checkpoint_load(kept, rows, width, out, dtype, stride, None)


def act_grad(lib, kept=FAR, rows=4, width=40, act=1, dy=2 * FAR, dtype=B.F32, stride=40, dx=3 * FAR, dx_stride=40):
    return lib.adasum_checkpoint_act_grad(kept, rows, width, act, dy, dtype, stride, dx, dx_stride, None)


def weight_grad(lib, kept=FAR, rows=4, width=40, dy=2 * FAR, dtype=B.F32, stride=16, outputs=16, grad=3 * FAR, grad_dtype=B.F32, offset=0,
                bias=640, accumulate=0, ws=4 * FAR, ws_bytes=1 << 30):
    return lib.adasum_checkpoint_weight_grad(kept, rows, width, dy, dtype, stride, outputs, grad, grad_dtype, offset, bias, accumulate, ws,
                                             ws_bytes, None)


@pytest.mark.parametrize("call, wrong", [
    (embedding, [dict(params=None), dict(ids=None), dict(out=None), dict(offset=-1), dict(rows=-1), dict(rows=0), dict(width=-1), dict(n=-1), dict(stride=7),
                 dict(stride=-8), dict(rows=1 << 31), dict(width=(1 << 24) + 1), dict(n=1 << 31), dict(offset=1 << 50)]),
    (embedding_grad, [dict(dy=None), dict(ids=None), dict(grad=None), dict(offset=-1), dict(rows=-1), dict(width=-1), dict(n=-1),
                      dict(stride=-1), dict(accumulate=2), dict(rows=1 << 31), dict(rows=(1 << 31) - 65536, width=1 << 24)]),
    (store, [dict(x=None), dict(kept=None), dict(rows=-1), dict(width=-1), dict(stride=-40), dict(rows=1 << 31), dict(width=1 << 25)]),
    (load, [dict(kept=None), dict(out=None), dict(rows=-1), dict(width=-1), dict(stride=39)]),
    (act_grad, [dict(kept=None), dict(dy=None), dict(dx=None), dict(rows=-1), dict(dx_stride=39), dict(stride=-1)]),
    (weight_grad, [dict(kept=None), dict(dy=None), dict(grad=None), dict(outputs=-1), dict(offset=-1), dict(accumulate=-1), dict(stride=-1),
                   dict(outputs=(1 << 24) + 1)]),
])
def test_invalid_arguments(lib, call, wrong):
    for kw in wrong:
        assert call(lib, **kw) == B.ERR_INVALID_ARG, kw


@pytest.mark.parametrize("call, wrong", [
    (embedding, [dict(dtype=9), dict(out_dtype=-1), dict(dtype=B.F64), dict(out_dtype=B.F64), dict(id_type=2)]),
    (embedding_grad, [dict(dtype=4), dict(grad_dtype=B.F64), dict(dtype=B.F64), dict(id_type=-1)]),
    (store, [dict(dtype=B.F64), dict(dtype=7)]),
    (load, [dict(dtype=B.F64), dict(dtype=-1)]),
    (act_grad, [dict(dtype=B.F64), dict(act=4), dict(act=-1)]),
    (weight_grad, [dict(dtype=B.F64, grad_dtype=B.F64), dict(grad_dtype=B.F64), dict(grad_dtype=5)]),
])
def test_unsupported_types(lib, call, wrong):
    for kw in wrong:
        assert call(lib, **kw) == B.ERR_UNSUPPORTED, kw


@pytest.mark.parametrize("call, names", [(embedding, ("params", "ids", "out")), (embedding_grad, ("dy", "ids", "grad")),
                                         (store, ("x", "kept")), (load, ("kept", "out")), (act_grad, ("kept", "dy", "dx")),
                                         (weight_grad, ("kept", "dy", "grad"))])
def test_misaligned_pointers(lib, call, names):
    for i, name in enumerate(names):
        assert call(lib, **{name: 9 * FAR + 8}) == B.ERR_MISALIGNED, name


def test_results_may_not_overlap_operands(lib):
    assert embedding(lib, out=FAR + 64) == B.ERR_ALIAS                       # 10 x 8 fp32 from FAR on
    assert embedding(lib, out=2 * FAR + 16) == B.ERR_ALIAS                   # the ids
    assert embedding_grad(lib, grad=FAR + 112) == B.ERR_ALIAS                # dy's last row
    assert embedding_grad(lib, grad=FAR - 320, offset=1) == B.ERR_ALIAS      # the layer's last element is dy's first
    assert embedding_grad(lib, grad=4 * FAR + 256) == B.ERR_ALIAS            # the workspace
    assert embedding_grad(lib, ws=FAR) == B.ERR_ALIAS
    assert store(lib, kept=FAR + 16) == B.ERR_ALIAS
    assert load(lib, out=FAR + 256) == B.ERR_ALIAS                           # the exponents, behind 4 x 64 bytes
    assert act_grad(lib, dx=2 * FAR + 16) == B.ERR_ALIAS                     # neither apart from dy nor dy itself
    assert act_grad(lib, dx=2 * FAR, dx_stride=48) == B.ERR_ALIAS            # dy itself, with other rows
    assert act_grad(lib, dx=FAR) == B.ERR_ALIAS
    assert weight_grad(lib, bias=639) == B.ERR_ALIAS                         # the weight's last element
    assert weight_grad(lib, grad=2 * FAR) == B.ERR_ALIAS
    assert weight_grad(lib, grad=FAR + 64) == B.ERR_ALIAS


def test_workspace_is_checked(lib):
    need = B.adasum_embedding_grad_workspace_bytes
    n = C.c_size_t(0)
    assert lib.adasum_embedding_grad_workspace_bytes(10, 8, 4, B.F32, C.byref(n)) == B.OK and n.value > 0
    assert embedding_grad(lib, ws_bytes=n.value - 1) == B.ERR_WORKSPACE
    assert embedding_grad(lib, ws=None) == B.ERR_WORKSPACE
    assert embedding_grad(lib, ws=4 * FAR + 16) == B.ERR_WORKSPACE
    assert lib.adasum_embedding_grad_workspace_bytes(10, 8, 4, 9, C.byref(n)) == B.ERR_UNSUPPORTED
    assert lib.adasum_embedding_grad_workspace_bytes(10, -8, 4, B.F32, C.byref(n)) == B.ERR_INVALID_ARG
    assert lib.adasum_embedding_grad_workspace_bytes(10, 8, 4, B.F32, None) == B.ERR_INVALID_ARG
    import torch
    assert need(0, 8, 4, torch.float32) == need(10, 0, 4, torch.float32) == need(10, 8, 0, torch.float32) == 0
    # a long sum into a small weight is cut, and the pieces need room
    assert lib.adasum_checkpoint_weight_grad_workspace_bytes(65536, 64, 64, B.BF16, C.byref(n)) == B.OK and n.value > 0
    assert weight_grad(lib, rows=65536, width=64, outputs=64, stride=64, dtype=B.BF16, bias=-1, ws_bytes=n.value - 1) == B.ERR_WORKSPACE
    assert weight_grad(lib, rows=65536, width=64, outputs=64, stride=64, dtype=B.BF16, bias=-1, ws=None) == B.ERR_WORKSPACE
    assert lib.adasum_checkpoint_weight_grad_workspace_bytes(4, 40, 16, B.F64, C.byref(n)) == B.ERR_UNSUPPORTED


def test_nothing_to_do_needs_no_device(lib):
    assert embedding(lib, n=0, ids=None, out=None, params=None) == B.OK
    assert embedding(lib, width=0, out=None, params=None) == B.OK
    assert embedding_grad(lib, rows=0, grad=None) == B.OK
    assert embedding_grad(lib, width=0, grad=None, dy=None) == B.OK
    assert embedding_grad(lib, n=0, dy=None, ids=None, ws=None, accumulate=1) == B.OK
    assert store(lib, rows=0, x=None, kept=None) == load(lib, width=0, kept=None, out=None) == B.OK
    assert act_grad(lib, rows=0, kept=None, dy=None, dx=None) == B.OK
    assert weight_grad(lib, outputs=0, dy=None, grad=None) == B.OK
    assert weight_grad(lib, width=0, kept=None, grad=None, bias=-1) == B.OK
    assert weight_grad(lib, width=0, kept=None) == B.ERR_INVALID_ARG          # a layer without inputs has no bias here


@pytest.mark.parametrize("rows, width, want", [(0, 5, 0), (3, 0, 0), (1, 1, 33), (2, 32, 66), (2, 33, 132), (7, 1023, 7 * 32 * 33)])
def test_checkpoint_bytes(lib, rows, width, want):
    n = C.c_size_t(1)
    assert lib.adasum_checkpoint_bytes(rows, width, C.byref(n)) == B.OK and n.value == want
    assert lib.adasum_checkpoint_bytes(-1, width, C.byref(n)) == B.ERR_INVALID_ARG
    assert lib.adasum_checkpoint_bytes(rows, width, None) == B.ERR_INVALID_ARG


def test_binding_refuses_what_is_not_on_a_device():
    import torch
    flat, ids = torch.zeros(80), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(ValueError):
        B.adasum_embedding(flat, 0, 10, 8, ids)
    with pytest.raises(ValueError):
        B.adasum_embedding_grad(torch.zeros(4, 8), ids, flat, 0, 10)
    with pytest.raises(ValueError):
        B.adasum_checkpoint_store(torch.zeros(4, 8))
    with pytest.raises(ValueError):
        B.Checkpoint(4, 40, torch.float64, device="cpu")
    with pytest.raises(ValueError):
        B.Checkpoint(4, 40, torch.float32, data=torch.zeros(10, dtype=torch.int8))
    kept = B.Checkpoint(4, 40, torch.float32, device="cpu")
    with pytest.raises(ValueError):
        B.adasum_checkpoint_act_grad(kept, torch.zeros(4, 40), "softplus")
    with pytest.raises(ValueError):
        B.adasum_checkpoint_weight_grad(kept, torch.zeros(4, 16), flat, 0)
