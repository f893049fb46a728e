"""Tensors of more than 2^31 elements through the dense operators, where only the tokens around and
behind that offset, and the last ones, have gradients: sums of whole numbers over them alone, exact in 32
bits, so that a token left out or read elsewhere shows whatever the length of the contraction."""
import sys

import pytest
import torch

from paper_2609_13846_amd import dtp
from tests.test_gpu_dense import DT, workspace
from tests.test_gpu_dense_tiles import product, whole

pytestmark = pytest.mark.gpu

K = 32


def far_tokens(T, per_token):
    """Forty tokens either side of element 2^31 of rows of `per_token`, and the last 71: an odd end."""
    at = 2 ** 31 // per_token
    assert at + 40 < T - 71
    return torch.cat((torch.arange(at - 40, at + 40), torch.arange(T - 71, T))).cuda()


def rows(T, at, values):
    """[T, ...] of zeros but for the tokens `at`."""
    out = torch.zeros(T, *values.shape[1:], dtype=values.dtype, device="cuda")
    out[at] = values
    return out


def zero_elsewhere(t, at):
    """Whether all rows but `at` are zeros, in pieces (of that many elements nothing else is made)."""
    t[at] = 0
    return all(not bool(p.any()) for p in t.split(8192))


@pytest.mark.parametrize("dtype,T,N", [("bf16", 290000, 8192), ("f32", 150000, 16384)])
def test_linear(dtype, T, N):
    print("[gpu] far linear", dtype, T, N, file=sys.stderr, flush=True)
    dt, code = DT[dtype]
    at = far_tokens(T, N)
    x, w, b = whole(1, 2, T, K).to(dt), whole(2, 2, N, K).to(dt), whole(3, 8, N).to(dt)
    some = whole(4, 2, at.numel(), N).to(dt)
    space = workspace(dtp.dtp_linear_workspace(T, K, N, code, backward=True))
    y, pre = torch.empty(T, N, dtype=dt, device="cuda"), torch.empty(T, N, device="cuda")
    dtp.dtp_linear_forward(T, K, N, code, x, w, y, bias=b, pre=pre, workspace=space)
    z = product(x[at], w) + b.double()
    assert torch.equal(pre[at].double(), z) and torch.equal(y[at], z.to(dt))
    del y, pre
    dy = rows(T, at, some)
    dx, dw, db = torch.empty_like(x), torch.empty_like(w), torch.empty_like(b)
    dtp.dtp_linear_backward(T, K, N, code, x, w, dy, dx=dx, dw=dw, dbias=db, workspace=space)
    assert torch.equal(dw, product(some.t(), x[at].t()).to(dt))
    assert torch.equal(db, some.double().sum(0).to(dt))
    assert torch.equal(dx[at], product(some, w.t()).to(dt)) and zero_elsewhere(dx, at)


@pytest.mark.parametrize("dtype,T,I", [("bf16", 140000, 8192), ("f32", 70000, 16384)])
def test_gated(dtype, T, I):
    """The kept pre-activations are the tensor of more than 2^31 elements."""
    print("[gpu] far gated", dtype, T, I, file=sys.stderr, flush=True)
    dt, code = DT[dtype]
    at = far_tokens(T, 2 * I)
    x, wg, wu = whole(1, 2, T, K).to(dt), whole(2, 2, I, K).to(dt), whole(3, 2, I, K).to(dt)
    space = workspace(dtp.dtp_gated_workspace(T, K, I, code, True))
    h, pre = torch.empty(T, I, dtype=dt, device="cuda"), torch.empty(T, 2, I, device="cuda")
    dtp.dtp_gated_forward(T, K, I, code, x, wg, wu, h, pre=pre, workspace=space)
    assert torch.equal(pre[at, 0].double(), product(x[at], wg)) and torch.equal(pre[at, 1].double(), product(x[at], wu))
    last = torch.empty(71, I, dtype=dt, device="cuda")
    dtp.dtp_gated_forward(71, K, I, code, x[T - 71:].clone(), wg, wu, last)
    assert torch.equal(h[T - 71:], last)
    # silu and its derivative are 0 and 1/2 at 0, and 128 and 1 at 128
    gate, up, some = 128.0 * (whole(4, 1, at.numel(), I) > 0), whole(5, 2, at.numel(), I), 2 * whole(6, 1, at.numel(), I)
    pre.zero_()
    pre[at, 0], pre[at, 1] = gate, up
    dg, du = some * up * torch.where(gate > 0, 1.0, 0.5), some * gate
    dh = h.zero_()
    dh[at] = some.to(dt)
    dx, dwg, dwu = torch.empty_like(x), torch.empty_like(wg), torch.empty_like(wu)
    dtp.dtp_gated_backward(T, K, I, code, x, wg, wu, pre, dh, dx=dx, dw_gate=dwg, dw_up=dwu, workspace=space)
    assert torch.equal(dwg, product(dg.t(), x[at].t()).to(dt)) and torch.equal(dwu, product(du.t(), x[at].t()).to(dt))
    assert torch.equal(dx[at], (product(dg, wg.t()) + product(du, wu.t())).to(dt)) and zero_elsewhere(dx, at)


def test_more_tiles_than_a_launch_takes():
    """2^28 fp32 tokens and some through 65 neurons: more than 2^22 tiles of 128 tokens x 64 neurons.
    x of 0 or 128, where silu is x exactly: h = 128 (128 w_up)."""
    T, I = 2 ** 28 + 70, 65
    print("[gpu] many tiles", T, I, file=sys.stderr, flush=True)
    x = torch.arange(T, dtype=torch.int32, device="cuda").remainder_(3).clamp_(max=1).float().mul_(128).view(T, 1)
    wg, wu = torch.ones(I, 1, device="cuda"), whole(1, 8, I, 1)
    h = torch.full((T, I), -1.0, device="cuda")
    dtp.dtp_gated_forward(T, 1, I, dtp.DTP_F32, x, wg, wu, h)
    assert all(torch.equal(a, b * (128 * wu.view(1, I))) for a, b in zip(h.split(1 << 22), x.split(1 << 22)))
