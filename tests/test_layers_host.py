"""CPU-only checks of the layer operators: bad arguments are refused before any CUDA call,
scratch sizes, and the tensor table's own checks."""
import ctypes

import pytest
import torch

from paper_2506_09092_b200 import binding as B
from paper_2506_09092_b200 import build as libbuild

P = 1 << 20             # a non-null, aligned stand-in address; never dereferenced on error


@pytest.fixture(scope="module", autouse=True)
def built():
    libbuild.build()


def ln(**k):
    a = dict(x=P, gamma=P, beta=P, y=P, mean=P, rstd=P, rows=4, n=8, ldx=8, ldy=8, dtype=B.BF16, param_dtype=B.F32,
             eps=1e-5)
    a.update(k)
    return B.layernorm_rows(**a, check=False)


def ln_bwd(**k):
    a = dict(dy=P, x=P, gamma=P, mean=P, rstd=P, dx=P, dgamma=P, dbeta=P, rows=4, n=8, lddy=8, ldx=8, lddx=8,
             dtype=B.BF16, param_dtype=B.BF16, scratch=P, scratch_bytes=1 << 30)
    a.update(k)
    return B.layernorm_rows_bwd(**a, check=False)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=3), B.ERR_INVALID_DTYPE), (dict(dtype=-1), B.ERR_INVALID_DTYPE),
    (dict(param_dtype=B.F16), B.ERR_INVALID_DTYPE), (dict(dtype=B.F32, param_dtype=B.BF16), B.ERR_INVALID_DTYPE),
    (dict(rows=-1), B.ERR_INVALID_DIM), (dict(n=-1), B.ERR_INVALID_DIM), (dict(rows=1 << 31), B.ERR_INVALID_DIM),
    (dict(n=1 << 31, ldx=1 << 31, ldy=1 << 31), B.ERR_INVALID_DIM), (dict(ldx=1 << 50), B.ERR_INVALID_DIM),
    (dict(ldx=7), B.ERR_INVALID_LD), (dict(ldy=7), B.ERR_INVALID_LD),
    (dict(eps=-1.0), B.ERR_INVALID_DIM), (dict(eps=float("nan")), B.ERR_INVALID_DIM),
    (dict(eps=float("inf")), B.ERR_INVALID_DIM),
    (dict(x=None), B.ERR_INVALID_POINTER), (dict(y=None), B.ERR_INVALID_POINTER),
    (dict(x=P + 1), B.ERR_MISALIGNED), (dict(gamma=P + 2), B.ERR_MISALIGNED), (dict(beta=P + 1), B.ERR_MISALIGNED),
    (dict(mean=P + 2), B.ERR_MISALIGNED), (dict(rstd=P + 1), B.ERR_MISALIGNED),
    (dict(rows=0, x=None, y=None), B.OK), (dict(n=0, x=None, y=None), B.OK),
])
def test_layernorm_rows_refusals(change, status):
    assert ln(**change) == status


@pytest.mark.parametrize("change,status", [
    (dict(dtype=3), B.ERR_INVALID_DTYPE), (dict(param_dtype=B.F16), B.ERR_INVALID_DTYPE),
    (dict(rows=-1), B.ERR_INVALID_DIM), (dict(n=-1), B.ERR_INVALID_DIM),
    (dict(lddy=7), B.ERR_INVALID_LD), (dict(ldx=7), B.ERR_INVALID_LD), (dict(lddx=7), B.ERR_INVALID_LD),
    (dict(dy=None), B.ERR_INVALID_POINTER), (dict(x=None), B.ERR_INVALID_POINTER),
    (dict(mean=None), B.ERR_INVALID_POINTER), (dict(rstd=None), B.ERR_INVALID_POINTER),
    (dict(dy=P + 1), B.ERR_MISALIGNED), (dict(dx=P + 1), B.ERR_MISALIGNED), (dict(dgamma=P + 1), B.ERR_MISALIGNED),
    (dict(scratch=None), B.ERR_WORKSPACE), (dict(scratch=P + 8), B.ERR_WORKSPACE),
    (dict(scratch_bytes=4 * 8 * 8 - 1), B.ERR_WORKSPACE),
    (dict(dx=None, dgamma=None, dbeta=None), B.OK), (dict(n=0, dy=None), B.OK),
    (dict(rows=0, dgamma=None, dbeta=None, dy=None, x=None), B.OK),
])
def test_layernorm_rows_bwd_refusals(change, status):
    assert ln_bwd(**change) == status


def test_layernorm_scratch_sizes():
    f = B.layernorm_rows_bwd_scratch_bytes
    assert f(4, 8) == 4 * 8 * 8 and f(0, 8) == 64 and f(4, 0) == 0
    assert f(-1, 8) == f(8, -1) == f(1 << 31, 8) == 0
    assert f(1 << 20, 4096) <= 148 * 2 * 4096 * 8 and f(1 << 20, 1 << 20) == 148 * 8 << 20


def table(*entries):
    class Table:
        count = len(entries)
        array = (B.CTensor * max(len(entries), 1))()
    for e, (data, out, n, dtype) in zip(Table.array, entries):
        e.data, e.out, e.n, e.dtype = data, out, n, dtype
    return Table


@pytest.mark.parametrize("entry,status", [
    ((P, P, -1, B.F32), B.ERR_INVALID_DIM), ((P, P, (1 << 40) + 1, B.F32), B.ERR_INVALID_DIM),
    ((P, P, 4, 3), B.ERR_INVALID_DTYPE), ((None, P, 4, B.F32), B.ERR_INVALID_POINTER),
    ((P + 2, P, 4, B.F32), B.ERR_MISALIGNED), ((P + 1, P, 4, B.F16), B.ERR_MISALIGNED),
])
def test_gradient_list_refusals(entry, status):
    t = table((P, P, 4, B.BF16), entry)
    assert B.grad_norm(t, P, P, 1 << 20, check=False) == status
    assert B.grad_clip(t, P, 1.0, check=False) == status
    assert B.grad_clip_norm(t, 1.0, 1e-6, P, P, 1 << 20, check=False) == status


def test_gradient_call_refusals():
    t = table((P, P, 4, B.BF16))
    need = B.grad_norm_scratch_bytes(1)
    assert need == B.grad_norm_scratch_bytes(0) == B.grad_norm_scratch_bytes(1024) < B.grad_norm_scratch_bytes(1025)
    assert B.grad_norm_scratch_bytes(-1) == 0
    assert B.grad_norm(t, None, P, need, check=False) == B.ERR_INVALID_POINTER
    assert B.grad_norm(t, P + 2, P, need, check=False) == B.ERR_MISALIGNED
    for scratch, size in ((None, need), (P + 8, need), (P, need - 1)):
        assert B.grad_norm(t, P, scratch, size, check=False) == B.ERR_WORKSPACE
        assert B.grad_clip_norm(t, 1.0, 1e-6, P, scratch, size, check=False) == B.ERR_WORKSPACE
    for bad in (-1.0, float("nan")):
        assert B.grad_clip(t, P, bad, check=False) == B.ERR_INVALID_DIM
        assert B.grad_clip(t, P, 1.0, bad, check=False) == B.ERR_INVALID_DIM
    out = table((P, None, 4, B.BF16))
    assert B.grad_clip(out, P, 1.0, check=False) == B.ERR_INVALID_POINTER
    assert B.grad_clip(table((P, P + 1, 4, B.BF16)), P, 1.0, check=False) == B.ERR_MISALIGNED
    assert B.lib().cudallm_grad_norm(None, 1, P, P, need, None) == B.ERR_INVALID_POINTER
    assert B.lib().cudallm_grad_norm(t.array, -1, P, P, need, None) == B.ERR_INVALID_DIM
    assert B.grad_clip(table((None, None, 0, B.F32)), P, 1.0, check=False) == B.OK       # nothing to scale


def test_host_tensors_are_refused_by_the_binding():
    x = torch.zeros(4, 8)
    with pytest.raises(TypeError):
        B.layernorm_rows(x, None, None, x, None, None, 4, 8, 8, 8, B.F32, B.F32)
    with pytest.raises(TypeError):
        B.tensor_table([x])


def test_struct_layout():
    assert ctypes.sizeof(B.CTensor) == 32


def xshape(**k):
    a = dict(batch=2, q_rows=5, kv_rows=7, q_heads=4, kv_heads=2, head_dim=64, dtype=B.BF16, scale=0.125,
             q_stride=(5 * 4 * 64, 4 * 64, 64), k_stride=(7 * 2 * 64, 2 * 64, 64), v_stride=(7 * 2 * 64, 2 * 64, 64),
             o_stride=(5 * 4 * 64, 4 * 64, 64))
    a.update(k)
    for f in ("q_stride", "k_stride", "v_stride", "o_stride"):
        a[f] = (ctypes.c_int64 * 3)(*a[f])
    return B.XattnShape(**a)


def fwd(shape, **k):
    a = dict(q=P, k=P, v=P, kv_lens=P, o=P, lse=P, scratch=P, scratch_bytes=1 << 40)
    a.update(k)
    return B.xattn_fwd(shape, check=False, **a)


def bwd(shape, **k):
    a = dict(q=P, k=P, v=P, kv_lens=P, o=P, lse=P, d_o=P, dq=P, dk=P, dv=P, scratch=P, scratch_bytes=1 << 40)
    a.update(k)
    return B.xattn_bwd(shape, check=False, **a)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=B.F32), B.ERR_INVALID_DTYPE), (dict(dtype=3), B.ERR_INVALID_DTYPE),
    (dict(batch=-1), B.ERR_INVALID_DIM), (dict(q_rows=-1), B.ERR_INVALID_DIM), (dict(kv_rows=1 << 31), B.ERR_INVALID_DIM),
    (dict(kv_heads=3), B.ERR_INVALID_DIM), (dict(kv_heads=0), B.ERR_INVALID_DIM),
    (dict(scale=-1.0), B.ERR_INVALID_DIM), (dict(scale=float("nan")), B.ERR_INVALID_DIM),
    (dict(scale=float("inf")), B.ERR_INVALID_DIM),
    (dict(head_dim=60), B.ERR_UNSUPPORTED_SHAPE), (dict(head_dim=136), B.ERR_UNSUPPORTED_SHAPE),
    (dict(q_stride=(1280, 256, 0)), B.ERR_INVALID_LD), (dict(q_stride=(1280, -256, 64)), B.ERR_INVALID_LD),
    (dict(k_stride=(896, 128, 56)), B.ERR_INVALID_LD),          # heads overlap
    (dict(v_stride=(840, 128, 64)), B.ERR_INVALID_LD),          # batch items overlap
    (dict(o_stride=(1284, 256, 64)), B.ERR_UNSUPPORTED_SHAPE),  # not a multiple of 8
    (dict(o_stride=(1 << 45, 256, 64)), B.ERR_INVALID_DIM),
    (dict(batch=0), B.OK), (dict(q_heads=0), B.OK), (dict(head_dim=0), B.OK),
])
def test_attention_shape_refusals(change, status):
    s = xshape(**change)
    assert fwd(s) == status and bwd(s) == status
    if status != B.OK:
        assert B.xattn_fwd_scratch_bytes(s) == B.xattn_bwd_scratch_bytes(s) == 0


def test_attention_operand_refusals():
    s = xshape()
    assert B.lib().cudallm_xattn_fwd(None, P, P, P, P, P, P, P, 1 << 30, None) == B.ERR_INVALID_POINTER
    for name in ("q", "k", "v", "o"):
        assert fwd(s, **{name: None}) == B.ERR_INVALID_POINTER
        assert fwd(s, **{name: P + 8}) == B.ERR_UNSUPPORTED_SHAPE
        assert bwd(s, **{name: None}) == B.ERR_INVALID_POINTER
        assert bwd(s, **{name: P + 8}) == B.ERR_UNSUPPORTED_SHAPE
    for name in ("kv_lens", "lse"):
        assert fwd(s, **{name: P + 2}) == B.ERR_MISALIGNED
        assert bwd(s, **{name: P + 2}) == B.ERR_MISALIGNED
    for name in ("lse", "d_o", "dq", "dk", "dv"):
        assert bwd(s, **{name: None}) == B.ERR_INVALID_POINTER
    for name in ("d_o", "dq", "dk", "dv"):
        assert bwd(s, **{name: P + 8}) == B.ERR_UNSUPPORTED_SHAPE
    need = B.xattn_bwd_scratch_bytes(s)
    assert need >= 2 * 4 * 5 * 4
    for scratch, size in ((None, need), (P + 8, need), (P, need - 1)):
        assert bwd(s, scratch=scratch, scratch_bytes=size) == B.ERR_WORKSPACE
    long = xshape(batch=1, q_rows=1, kv_rows=1 << 16, k_stride=(0, 128, 64), v_stride=(0, 128, 64))
    need = B.xattn_fwd_scratch_bytes(long)
    assert need > 0
    for scratch, size in ((None, need), (P + 8, need), (P, need - 1)):
        assert fwd(long, scratch=scratch, scratch_bytes=size) == B.ERR_WORKSPACE
    assert fwd(xshape(q_rows=0), q=None, k=None, v=None, o=None) == B.OK
    assert bwd(xshape(q_rows=0), q=None, o=None, lse=None, d_o=None, dq=None, dk=None, dv=None, scratch=None) == B.OK
    assert bwd(xshape(q_rows=0, kv_rows=0), q=None, k=None, v=None) == B.OK


def test_attention_shape_from_tensors():
    q = torch.zeros(2, 5, 4, 64, dtype=torch.bfloat16)
    kv = torch.zeros(2, 7, 2, 2, 64, dtype=torch.bfloat16)
    s = B.XattnShape.of(q, kv[:, :, 0], kv[:, :, 1], q)
    assert (s.batch, s.q_rows, s.kv_rows, s.q_heads, s.kv_heads, s.head_dim) == (2, 5, 7, 4, 2, 64)
    assert list(s.k_stride) == [7 * 4 * 64, 4 * 64, 64] and s.scale == 0.125 and s.dtype == B.BF16
    for bad in ((q.float(), kv[:, :, 0], kv[:, :, 1], q), (q.float(),) * 4):
        with pytest.raises(TypeError):
            B.XattnShape.of(*bad)
    for bad in ((q, kv[:, :, 0], kv[:, :1, 1], q), (q, kv[:, :, 0], kv[:, :, 1], q[:, :4]), (q.transpose(2, 3),) * 4):
        with pytest.raises(ValueError):
            B.XattnShape.of(*bad)
    assert ctypes.sizeof(B.XattnShape) == 152
