"""CPU-only: what the binding of the layer operators refuses of the tensors themselves, before any CUDA call.  The
tensors here lie in host memory, so a call whose layouts are in order ends at the check after them."""
import ctypes

import pytest
import torch

from paper_2506_09092_b200 import binding as B

BF, H = torch.bfloat16, torch.float16


def operands(t=BF):
    """Queries (2, 5, 4, 64); keys and values of 7 states and 2 heads side by side in one tensor."""
    q = torch.zeros(2, 5, 4, 64, dtype=t)
    kv = torch.zeros(2, 7, 2, 2, 64, dtype=t)
    a = dict(q=q, k=kv[:, :, 0], v=kv[:, :, 1], kv_lens=torch.tensor([7, 3], dtype=torch.int32), o=torch.zeros_like(q),
             lse=torch.zeros(2, 4, 5))
    return B.XattnShape.of(a["q"], a["k"], a["v"], a["o"]), a


def gradients(a):
    dkv = torch.zeros(2, 7, 2, 2, 64, dtype=a["q"].dtype)
    return dict(a, d_o=torch.zeros_like(a["o"]), dq=torch.zeros_like(a["q"]), dk=dkv[:, :, 0], dv=dkv[:, :, 1])


def fwd(shape, a):
    B.xattn_fwd(shape, scratch=None, scratch_bytes=0, **a)


def bwd(shape, a):
    B.xattn_bwd(shape, scratch=None, scratch_bytes=0, **a)


def passes_the_layouts(call, shape, a):
    with pytest.raises(TypeError, match="host memory"):
        call(shape, a)


@pytest.mark.parametrize("t", [BF, H])
def test_operands_as_the_shape_says(t):
    shape, a = operands(t)
    passes_the_layouts(fwd, shape, a)
    passes_the_layouts(fwd, shape, dict(a, kv_lens=None, lse=None))
    g = gradients(a)
    passes_the_layouts(bwd, shape, g)
    passes_the_layouts(bwd, shape, dict(g, dk=None, dv=None))
    # flat buffers, and heads x rows buffers behind a transposed view, hold what the strides address
    passes_the_layouts(fwd, shape, dict(a, q=a["q"].reshape(10, 256), o=torch.zeros(10 * 256 + 9, dtype=t), lse=torch.zeros(99)))
    wide = torch.zeros(2, 4, 5, 64, dtype=t)
    turned = B.XattnShape.of(wide.transpose(1, 2), a["k"], a["v"], a["o"])
    passes_the_layouts(fwd, turned, dict(a, q=wide))
    passes_the_layouts(fwd, turned, dict(a, q=wide.transpose(1, 2)))


@pytest.mark.parametrize("name", ["dq", "dk", "dv", "d_o", "o", "q", "k", "v"])
def test_a_result_or_operand_of_other_strides_is_refused(name):
    """The one that comes by itself: torch.empty_like of a part of a larger tensor is compact, and half as long
    as the strides of that part reach."""
    shape, a = operands()
    g = gradients(a)
    other = torch.empty_like(g[name]) if name in ("dk", "dv", "k", "v") else g[name].transpose(1, 2).contiguous().transpose(1, 2)
    assert other.shape == g[name].shape and other.stride() != g[name].stride()
    with pytest.raises(ValueError, match=f"{name} has strides"):
        bwd(shape, dict(g, **{name: other}))
    if name in a:
        with pytest.raises(ValueError, match=f"{name} has strides"):
            fwd(shape, dict(a, **{name: other}))


@pytest.mark.parametrize("name", ["dq", "dk", "dv", "d_o", "o", "q", "k", "v"])
def test_operands_of_other_types_or_too_short_are_refused(name):
    shape, a = operands()
    g = gradients(a)
    for other, error in ((g[name].half(), TypeError), (g[name].float(), TypeError), (g[name][:, :-1], ValueError),
                         (g[name][:1], ValueError), (torch.zeros(100, dtype=BF), ValueError), (torch.zeros(0, dtype=BF), ValueError)):
        for call, args in ((fwd, a), (bwd, g)):
            if name in args:
                with pytest.raises(error, match=f"^{name}"):
                    call(shape, dict(args, **{name: other}))


def test_lengths_and_lse_of_other_types_are_refused():
    shape, a = operands()
    bad = [("kv_lens", torch.tensor([7, 3]), TypeError), ("kv_lens", torch.tensor([7.0, 3.0]), TypeError),
           ("kv_lens", torch.tensor([7], dtype=torch.int32), ValueError),
           ("kv_lens", torch.zeros(4, dtype=torch.int32)[::2], ValueError),
           ("lse", torch.zeros(2, 4, 5, dtype=BF), TypeError), ("lse", torch.zeros(2, 4, 4), ValueError),
           ("lse", torch.zeros(2, 5, 4).transpose(1, 2), ValueError), ("lse", torch.zeros(2, 4, 5, dtype=torch.float64), TypeError)]
    for name, t, error in bad:
        for call, args in ((fwd, a), (bwd, gradients(a))):
            with pytest.raises(error, match=f"^{name}"):
                call(shape, dict(args, **{name: t}))


def test_a_changed_shape_is_looked_at_anew():
    shape, a = operands()
    passes_the_layouts(fwd, shape, a)
    shape.kv_rows = 8
    with pytest.raises(ValueError, match="^k"):
        fwd(shape, a)
    shape.kv_rows = 6                                      # the first six states of longer tensors
    passes_the_layouts(fwd, shape, a)
    shape.k_stride[1] = 512
    with pytest.raises(ValueError, match="^k"):
        fwd(shape, a)
    shape.k_stride[1] = 256
    shape.dtype = B.F16
    with pytest.raises(TypeError, match="^q"):
        fwd(shape, a)


def test_sizes_of_one_or_none_may_have_any_strides():
    q = torch.zeros(1, 1, 4, 64, dtype=BF)
    k = torch.zeros(1, 9, 4, 64, dtype=BF)
    shape = B.XattnShape.of(q, k, k, q)
    odd = torch.as_strided(q, q.shape, (7, 3, 64, 1))
    passes_the_layouts(fwd, shape, dict(q=odd, k=k, v=k, kv_lens=None, o=odd, lse=None))
    none = torch.zeros(1, 0, 4, 64, dtype=BF)
    shape = B.XattnShape.of(q, none, none, q)
    passes_the_layouts(fwd, shape, dict(q=q, k=torch.zeros(0, dtype=BF), v=none.float(), kv_lens=None, o=q, lse=None))


def test_addresses_and_refusals_of_the_call_itself_are_as_before():
    P = 1 << 20
    shape, _ = operands()
    bad = B.XattnShape.from_buffer_copy(shape)
    bad.dtype = 3
    zeros = torch.zeros(4)
    with pytest.raises(TypeError, match="host memory"):
        B.xattn_fwd(bad, zeros, zeros, zeros, None, zeros, None, None, 0)
    assert B.xattn_fwd(bad, P, P, P, P, P, P, None, 0, check=False) == B.ERR_INVALID_DTYPE
    assert B.xattn_fwd(None, P, P, P, P, P, P, None, 0, check=False) == B.ERR_INVALID_POINTER
    assert B.xattn_bwd(ctypes.pointer(bad), *[P] * 11, P, 0, check=False) == B.ERR_INVALID_DTYPE
