"""Argument checks of the dense operators that need no GPU: sizes, types, what must be given
together, workspace sizes; and the reference's formulas against torch's derivatives."""
import pytest
import torch

from paper_2609_13846_amd import dtp
from tests import dense_reference as ref

BF16, F32 = dtp.DTP_BF16, dtp.DTP_F32
INVALID, UNSUPPORTED = dtp.DTP_ERR_INVALID_ARG, dtp.DTP_ERR_UNSUPPORTED
P = 1 << 20  # an address that no call may get as far as reading


def expect(status, fn, *a, **k):
    with pytest.raises(dtp.DtpError) as e:
        fn(*a, **k)
    assert e.value.status == status and str(e.value)


@pytest.mark.parametrize("T,K,N,dtype,status", [(-1, 8, 8, BF16, INVALID), (1, 0, 8, BF16, INVALID), (1, 8, -3, F32, INVALID),
                                                (1, 8, 8, 2, UNSUPPORTED), (1, 1 << 21, 8, BF16, UNSUPPORTED),
                                                (1, 1 << 20, 1 << 12, BF16, UNSUPPORTED), ((1 << 30) + 1, 8, 8, BF16, UNSUPPORTED)])
def test_sizes_and_types(T, K, N, dtype, status):
    expect(status, dtp.dtp_linear_forward, T, K, N, dtype, P, P, P)
    expect(status, dtp.dtp_linear_backward, T, K, N, dtype, P, P, P, dx=P)
    expect(status, dtp.dtp_gated_forward, T, K, N, dtype, P, P, P, P)
    expect(status, dtp.dtp_gated_backward, T, K, N, dtype, P, P, P, P, P, dx=P)
    assert dtp.dtp_linear_workspace(T, K, N, dtype) == -1
    assert dtp.dtp_gated_workspace(T, K, N, dtype) == -1
    assert dtp.lib().dtp_last_error()


def test_activations_and_alpha():
    expect(UNSUPPORTED, dtp.dtp_linear_forward, 1, 8, 8, BF16, P, P, P, act=3)
    expect(UNSUPPORTED, dtp.dtp_gated_forward, 1, 8, 8, BF16, P, P, P, P, act=dtp.DTP_ACT_NONE)
    expect(UNSUPPORTED, dtp.dtp_gated_backward, 1, 8, 8, BF16, P, P, P, P, P, dx=P, act=-1)
    assert dtp.dtp_linear_workspace(4, 8, 8, BF16, 5) == -1
    for alpha in (float("nan"), float("inf")):
        expect(INVALID, dtp.dtp_linear_forward, 1, 8, 8, BF16, P, P, P, alpha=alpha)
        expect(INVALID, dtp.dtp_linear_backward, 1, 8, 8, BF16, P, P, P, dx=P, alpha=alpha)


def test_missing_arguments():
    lib = dtp.lib()
    assert lib.dtp_linear_forward(1, 8, 8, BF16, None, P, None, None, 0, 1.0, P, None, None, 0, None) == INVALID
    assert lib.dtp_linear_forward(1, 8, 8, BF16, P, P, None, None, 0, 1.0, None, None, None, 0, None) == INVALID
    assert lib.dtp_gated_forward(1, 8, 8, BF16, P, P, None, 1, P, None, None, 0, None) == INVALID
    # dx needs the weight, dw the input, an activation z
    assert lib.dtp_linear_backward(1, 8, 8, BF16, P, None, P, 0, 1.0, None, P, None, None, None, 0, None) == INVALID
    assert lib.dtp_linear_backward(1, 8, 8, BF16, None, P, P, 0, 1.0, None, None, P, None, None, 0, None) == INVALID
    assert lib.dtp_linear_backward(1, 8, 8, BF16, P, P, P, 1, 1.0, None, P, None, None, None, 0, None) == INVALID
    assert lib.dtp_gated_backward(1, 8, 8, BF16, P, P, P, 1, P, P, None, P, None, None, 0, None) == INVALID  # one dw
    # nothing asked for is nothing done
    assert lib.dtp_linear_backward(1, 8, 8, BF16, None, None, None, 0, 1.0, None, None, None, None, None, 0, None) == 0
    with pytest.raises(ValueError, match="required"):
        dtp.dtp_linear_backward(1, 8, 8, BF16, P, P, P, dx=P, act=dtp.DTP_ACT_SILU)


def test_no_tokens_is_a_no_op_before_any_gpu_work():
    dtp.dtp_linear_forward(0, 8, 8, BF16, 0, 0, 0)
    dtp.dtp_gated_forward(0, 8, 8, F32, 0, 0, 0, 0)


def test_host_memory_and_odd_addresses_are_refused():
    expect(INVALID, dtp.dtp_linear_forward, 1, 8, 8, BF16, P + 2, P, P)
    x = torch.ones(4, 8, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="on the GPU"):
        dtp.dtp_linear_forward(4, 8, 8, BF16, x, x, x)
    with pytest.raises(TypeError, match="workspace"):
        dtp.dtp_linear_forward(1, 8, 8, BF16, P, P, P, workspace=P)


def overlaps(status, name):
    return status == INVALID and dtp.lib().dtp_last_error().decode().endswith(name)


def test_an_output_is_in_place_of_one_input_only():
    """y may be the residual, but not where that is x too, which other blocks still read; so for the heads."""
    lib, far = dtp.lib(), P + (1 << 16)
    assert overlaps(lib.dtp_linear_forward(4, 8, 8, BF16, P, far, None, P, 0, 1.0, P, None, None, 0, None), "y overlaps x")
    assert overlaps(lib.dtp_linear_forward(4, 8, 8, BF16, far, P, None, P, 0, 1.0, P, None, None, 0, None), "y overlaps w")
    q, k, o, gamma, pos = (P + (i << 16) for i in range(5))

    def forward(q, k, q_out, k_out):
        return lib.dtp_qk_norm_rotate_forward(2, 2, 2, 64, BF16, q, 128, k, 128, gamma, gamma, 1e-6, pos, gamma, 64, q_out, k_out,
                                              None)

    def backward(dq_out, dk_out, dq, dk):
        return lib.dtp_qk_norm_rotate_backward(2, 2, 2, 64, BF16, q, 128, k, 128, gamma, gamma, 1e-6, pos, gamma, 64, dq_out,
                                               dk_out, dq, dk, None, None, None, 0, None)
    assert overlaps(forward(q, q, q, o), "q_out overlaps k")
    assert overlaps(forward(q, k, k, o), "q_out overlaps k")
    assert overlaps(forward(k, k, o, k), "k_out overlaps q")
    assert overlaps(backward(o, o, o, o + 512), "dq overlaps dk_out")
    assert overlaps(backward(q, o, q, o + 512), "dq overlaps q")
    assert overlaps(backward(o, o + 512, o + 1024, o), "dk overlaps dq_out")


def test_workspace_sizes():
    """Enough for the backward pass is enough for the forward one; sizes do not shrink with it."""
    for T in (0, 1, 16, 100, 4096, 65536):
        for dtype in (BF16, F32):
            for K, N in ((1024, 1024), (1040, 2810), (33, 7)):
                f = dtp.dtp_linear_workspace(T, K, N, dtype)
                assert 0 <= f <= dtp.dtp_linear_workspace(T, K, N, dtype, dtp.DTP_ACT_SILU, True)
                f = dtp.dtp_gated_workspace(T, K, N, dtype)
                assert 0 <= f <= dtp.dtp_gated_workspace(T, K, N, dtype, True)


QK = dict(n_tokens=2, n_q_heads=4, n_kv_groups=2, head_dim=64, dtype=BF16)


def qk_forward(q_stride=256, k_stride=128, gq=P, gk=P, eps=1e-6, pos=P, inv=P, rot=64, q=P, k=P, out=P, **kw):
    a = {**QK, **kw}
    return dtp.lib().dtp_qk_norm_rotate_forward(a["n_tokens"], a["n_q_heads"], a["n_kv_groups"], a["head_dim"], a["dtype"], q,
                                                q_stride, k, k_stride, gq, gk, eps, pos, inv, rot, out, out, None)


@pytest.mark.parametrize("kw,status", [
    (dict(n_tokens=-1), INVALID), (dict(n_q_heads=0), INVALID), (dict(n_kv_groups=3), INVALID), (dict(head_dim=63), INVALID),
    (dict(head_dim=258, q_stride=4096, k_stride=4096), UNSUPPORTED), (dict(dtype=9), UNSUPPORTED), (dict(gk=None), INVALID),
    (dict(pos=None), INVALID), (dict(inv=None), INVALID), (dict(rot=0), INVALID), (dict(rot=66), INVALID),
    (dict(rot=33), INVALID), (dict(rot=-2), INVALID), (dict(gq=None, gk=None, pos=None, inv=None, rot=0), INVALID),
    (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(q_stride=255), INVALID), (dict(k_stride=0), INVALID),
    (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(out=None), INVALID),
])
def test_qk_arguments(kw, status):
    assert qk_forward(**kw) == status
    assert dtp.lib().dtp_last_error()


def test_qk_backward_arguments_and_workspace():
    def back(dgq, dgk, gq=P, dq=P):
        return dtp.lib().dtp_qk_norm_rotate_backward(2, 4, 2, 64, BF16, P, 256, P, 128, gq, gq, 1e-6, P, P, 64, P, P, dq, P,
                                                     dgq, dgk, None, 0, None)
    assert back(P, None) == INVALID
    assert back(P, P, gq=None) == INVALID  # no norm, no dgamma
    assert back(None, None, dq=None) == INVALID
    assert dtp.dtp_qk_norm_rotate_workspace(0, 4, 2, 64, BF16) == 0
    assert 0 < dtp.dtp_qk_norm_rotate_workspace(5, 4, 2, 64, BF16) <= dtp.dtp_qk_norm_rotate_workspace(1 << 20, 4, 2, 64, BF16)
    assert dtp.dtp_qk_norm_rotate_workspace(5, 4, 3, 64, BF16) == -1


def test_qk_binding_checks_the_strides():
    q = torch.zeros(4, 2, 8, dtype=torch.bfloat16)
    with pytest.raises(TypeError, match="3 dimensions"):
        dtp._heads(q[0], "q", ("bfloat16",), 4, 2, 8)
    with pytest.raises(ValueError, match="shape"):
        dtp._heads(q, "q", ("bfloat16",), 4, 2, 16)
    with pytest.raises(ValueError, match="contiguous"):
        dtp._heads(q.transpose(1, 2), "q", ("bfloat16",), 4, 8, 2)
    with pytest.raises(ValueError, match="on the GPU"):
        dtp._heads(q, "q", ("bfloat16",), 4, 2, 8)
    with pytest.raises(ValueError, match="together"):
        dtp._rotation(q, None, 4)


def test_reference_gradients_are_the_derivatives():
    """The formulas that the GPU tests compare with, against torch's derivatives in 64 bits."""
    g = torch.Generator().manual_seed(0)

    def leaf(*shape):
        return torch.randn(*shape, generator=g).requires_grad_()

    x, w, wu, b, dy = leaf(5, 6), leaf(7, 6), leaf(7, 6), leaf(7), torch.randn(5, 7, generator=g)
    for name, f in (("silu", torch.nn.functional.silu), ("gelu", lambda z: torch.nn.functional.gelu(z, approximate="tanh"))):
        z = x.double() @ w.double().t() + b.double()
        gx, gw, gb = torch.autograd.grad(1.5 * f(z), (x, w, b), dy.double())
        got = ref.linear_grads(x.detach(), w.detach(), dy, z.detach(), torch.zeros_like(z), name, 1.5)
        for k, v in (("dx", gx), ("dw", gw), ("db", gb)):
            assert torch.allclose(got[k][0], v.double(), rtol=1e-5, atol=1e-5)
        xd = x.double()
        h = f(xd @ w.double().t()) * (xd @ wu.double().t())
        grads = torch.autograd.grad(h, (x, w, wu), dy.double())
        _, _, kept = ref.gated(x.detach(), w.detach(), wu.detach(), name)
        got = ref.gated_grads(x.detach(), w.detach(), wu.detach(), dy, kept, name)
        for k, v in zip(("dx", "dw_gate", "dw_up"), grads):
            assert torch.allclose(got[k][0], v.double(), rtol=1e-5, atol=1e-5)
    v, gamma, dout = leaf(4, 3, 12), leaf(12), torch.randn(4, 3, 12, generator=g)
    pos, inv = torch.tensor([0, 5, -7, 100000], dtype=torch.int32), torch.tensor([1.0, 0.3, 0.01])
    out, _ = ref.qk(v, gamma, 1e-6, pos, inv)
    gv, gg = torch.autograd.grad(out, (v, gamma), dout.double())
    got = ref.qk_grads(v.detach(), gamma.detach(), 1e-6, pos, inv, dout)
    assert torch.allclose(got["d"][0], gv.double(), rtol=1e-5, atol=1e-5)
    assert torch.allclose(got["dgamma"][0], gg.double(), rtol=1e-5, atol=1e-5)
