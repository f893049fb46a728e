"""Norms of heads whose squares leave the range of 32 bits, beside heads whose squares do not."""
import sys

import pytest
import torch

from paper_2609_13846_amd import dtp
from tests import dense_reference as ref
from tests.test_gpu_dense import DT, normal, workspace
from tests.test_gpu_qk_norm import frequencies

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh,offset", [(128, 0), (130, 1), (64, 0)])
@pytest.mark.parametrize("eps", [1e-6, 0.0])
def test_heads_of_any_size(dtype, dh, offset, eps):
    """Heads of 1e19 (where a sum of squares leaves the range, its terms do not), 1e25 and 1e37; of 1e-19,
    where squares lose bits, and 1e-25, where they are nothing; each with a neighbour of unit size.  The
    bounds are those of every other head: the norm of a head does not depend on its scale, but for eps."""
    T, H, G = 6, 4, 2
    dt, code = DT[dtype]
    print("[gpu] qk range", dtype, dh, offset, eps, file=sys.stderr, flush=True)
    flat = normal(1, T * (H + G) * dh + offset, scale=2.0)[offset:].view(T, H + G, dh)
    for t, size in enumerate((1e19, 1e25, 1e37, 1e-19, 1e-25)):
        flat[t, t % H] *= size
        flat[t, H + t % G] *= size
    v = torch.empty(T * (H + G) * dh + offset, dtype=dt, device="cuda")[offset:]
    v.copy_(flat.reshape(-1))
    rows = v.view(T, H + G, dh)
    q, k = rows[:, :H], rows[:, H:]
    assert bool(torch.isfinite(q).all())
    gamma = [(1 + normal(2 + i, dh, scale=0.2)).to(dt) for i in range(2)]
    pos, inv = torch.arange(T, dtype=torch.int32, device="cuda") * 997, frequencies(dh)
    dq_out, dk_out = normal(5, T, H, dh, dtype=dt), normal(6, T, G, dh, dtype=dt)
    out = [torch.empty_like(t) for t in (dq_out, dk_out)]
    grad = [torch.empty_like(t) for t in out]
    dgamma = [torch.empty_like(t) for t in gamma]
    common = dict(gamma_q=gamma[0], gamma_k=gamma[1], eps=eps, positions=pos, inv_freq=inv)
    dtp.dtp_qk_norm_rotate_forward(T, H, G, dh, code, q, k, *out, **common)
    dtp.dtp_qk_norm_rotate_backward(T, H, G, dh, code, q, k, dq_out, dk_out, *grad, dgamma_q=dgamma[0], dgamma_k=dgamma[1],
                                    workspace=workspace(dtp.dtp_qk_norm_rotate_workspace(T, H, G, dh, code)), **common)
    torch.cuda.synchronize()
    for i, (x, d) in enumerate(((q, dq_out), (k, dk_out))):
        ref.check(out[i], *ref.qk(x, gamma[i], eps, pos, inv), "q" if i == 0 else "k")
        want = ref.qk_grads(x, gamma[i], eps, pos, inv, d)
        ref.check(grad[i], *want["d"], "d")
        ref.check(dgamma[i], *want["dgamma"], "dgamma")


def test_infinite_heads_are_nan_alone():
    """Infinity over infinity is NaN in the formula; so in the head's own results only."""
    T, H, G, dh = 3, 4, 4, 64
    q, k = normal(1, T, H, dh), normal(2, T, G, dh)
    q[1, 2, 5] = float("inf")
    gamma, out, k_out = torch.ones(dh, device="cuda"), torch.empty_like(q), torch.empty_like(k)
    dtp.dtp_qk_norm_rotate_forward(T, H, G, dh, dtp.DTP_F32, q, k, out, k_out, gamma_q=gamma, gamma_k=gamma)
    nan = torch.isnan(out)
    assert bool(nan[1, 2, 5]) and int(nan.sum()) == 1  # the others are finite over infinity
    assert not bool(out[1, 2, :5].any()) and bool(torch.isfinite(k_out).all())
