"""The per-head norms with the rotation by position against their formulas in 64 bits, element by
element (tests/dense_reference.py derives the bounds): head widths, partial rotations, slices of a
packed projection at any alignment, far and negative positions, in place, gradients."""
import sys

import pytest
import torch

from paper_2609_13846_amd import dtp
from tests import dense_reference as ref
from tests.test_gpu_dense import DT, GUARD, Out, normal, refused, workspace

pytestmark = pytest.mark.gpu


def announce(*a):
    print("[gpu]", *a, file=sys.stderr, flush=True)


def frequencies(rot):
    if not rot:
        return None
    return (1e4 ** (-torch.arange(rot // 2, dtype=torch.float64) * 2 / rot)).float().cuda()


def run(T, H, G, dh, dtype, norm=True, rot=None, packed=True, offset=0, extra=0, seed=0, positions=None, eps=1e-6, zero=()):
    dt, code = DT[dtype]
    rot = dh if rot is None else rot
    width = (H + 2 * G) * dh + extra
    flat = normal(seed, T * width + offset, scale=2.0, dtype=dt)
    rows = flat[offset:].view(T, width)
    q, k = rows[:, :H * dh].view(T, H, dh), rows[:, H * dh:(H + G) * dh].view(T, G, dh)
    if not packed:
        q, k = q.contiguous(), k.contiguous()
    for t, h in zero:
        q[t, h] = 0
    gq, gk = ((1 + normal(seed + i, dh, scale=0.2)).to(dt) if norm else None for i in (1, 2))
    inv = frequencies(rot)
    if rot and positions is None:
        g = torch.Generator(device="cuda").manual_seed(seed + 3)
        positions = torch.randint(0, 40000, (T,), generator=g, device="cuda", dtype=torch.int32)
    dq_out, dk_out = normal(seed + 4, T, H, dh, dtype=dt), normal(seed + 5, T, G, dh, dtype=dt)
    o = dict(q=Out(T, H, dh, dtype=dt), k=Out(T, G, dh, dtype=dt), dq=Out(T, H, dh, dtype=dt), dk=Out(T, G, dh, dtype=dt),
             dgq=Out(dh, dtype=dt), dgk=Out(dh, dtype=dt))
    ws = workspace(dtp.dtp_qk_norm_rotate_workspace(T, H, G, dh, code))
    common = dict(gamma_q=gq, gamma_k=gk, eps=eps, positions=positions, inv_freq=inv)
    dtp.dtp_qk_norm_rotate_forward(T, H, G, dh, code, q, k, o["q"].t, o["k"].t, **common)
    dtp.dtp_qk_norm_rotate_backward(T, H, G, dh, code, q, k, dq_out, dk_out, o["dq"].t, o["dk"].t,
                                    dgamma_q=o["dgq"].t if norm else None, dgamma_k=o["dgk"].t if norm else None,
                                    workspace=ws, **common)
    torch.cuda.synchronize()
    assert all(v.untouched() for v in o.values())
    return dict(q=q, k=k, dq_out=dq_out, dk_out=dk_out, common=common, out={n: v.t for n, v in o.items()})


def check(v):
    c, out = v["common"], v["out"]
    for n in ("q", "k"):
        gamma = c["gamma_" + n]
        value, bound = ref.qk(v[n], gamma, c["eps"], c["positions"], c["inv_freq"])
        ref.check(out[n], value, bound, n)
        grads = ref.qk_grads(v[n], gamma, c["eps"], c["positions"], c["inv_freq"], v["d%s_out" % n])
        ref.check(out["d" + n], *grads["d"], "d" + n)
        if gamma is not None:
            ref.check(out["dg" + n], *grads["dgamma"], "dgamma_" + n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dh,rot", [(2, 2), (2, 0), (6, 2), (16, 16), (30, 10), (64, 64), (64, 32), (80, 80), (80, 40), (96, 96),
                                    (112, 112), (128, 128), (128, 0), (128, 2), (130, 130), (254, 254), (256, 256), (256, 64)])
def test_widths(dtype, dh, rot):
    for T, H, G in ((1, 1, 1), (7, 6, 2), (33, 9, 3)):
        announce("qk", dtype, dh, rot, T, H, G)
        check(run(T, H, G, dh, dtype, rot=rot, seed=dh))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,H,G,dh", [(1, 16, 8, 128), (4, 32, 8, 128), (5, 40, 1, 64), (1000, 16, 8, 96), (4099, 4, 4, 32),
                                      (5000, 12, 3, 80)])
def test_tokens_and_heads(dtype, T, H, G, dh):
    announce("qk", dtype, T, H, G, dh)
    check(run(T, H, G, dh, dtype, seed=T))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("packed,offset,extra", [(False, 0, 0), (True, 1, 0), (True, 2, 4), (True, 0, 3), (True, 4, 8)])
def test_rows_at_any_address(dtype, packed, offset, extra):
    """Slices of a packed projection whose rows start at odd elements, or lie an odd number apart."""
    check(run(50, 8, 4, 64, dtype, packed=packed, seed=1, offset=offset, extra=extra))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rotation_alone(dtype):
    check(run(65, 6, 2, 96, dtype, norm=False))
    check(run(3, 6, 2, 96, dtype, norm=False, rot=48))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_and_negative_positions(dtype):
    pos = torch.tensor([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 1000003, -999999, 16777217], dtype=torch.int32, device="cuda")
    check(run(8, 4, 2, 128, dtype, positions=pos))


def test_zero_heads_and_no_eps():
    """A head of zeros is zeros with any eps > 0 and its gradient that of eps; with eps = 0 it is
    NaN as the formula is, and its neighbours are not."""
    v = run(6, 4, 2, 64, "f32", zero=((2, 1),), eps=1e-2)
    check(v)
    assert not bool(v["out"]["q"][2, 1].any())
    v = run(6, 3, 1, 64, "f32", zero=((2, 1),), eps=0.0)  # three heads: lanes of a fourth are idle
    assert bool(torch.isnan(v["out"]["q"][2, 1]).all())
    keep = torch.ones(6, 3, dtype=torch.bool, device="cuda")
    keep[2, 1] = False
    value, bound = ref.qk(v["q"], v["common"]["gamma_q"], 0.0, v["common"]["positions"], v["common"]["inv_freq"])
    ref.check(v["out"]["q"][keep], value[keep], bound[keep], "the others")
    grads = ref.qk_grads(v["k"], v["common"]["gamma_k"], 0.0, v["common"]["positions"], v["common"]["inv_freq"], v["dk_out"])
    ref.check(v["out"]["dgk"], *grads["dgamma"], "dgamma_k")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place(dtype):
    dt, code = DT[dtype]
    v = run(40, 6, 3, 128, dtype, packed=False)
    q, k, dq, dk = (v[n].clone() for n in ("q", "k", "dq_out", "dk_out"))
    dtp.dtp_qk_norm_rotate_backward(40, 6, 3, 128, code, v["q"], v["k"], dq, dk, dq, dk, **v["common"])
    dtp.dtp_qk_norm_rotate_forward(40, 6, 3, 128, code, q, k, q, k, **v["common"])
    for a, n in ((q, "q"), (k, "k"), (dq, "dq"), (dk, "dk")):
        assert torch.equal(a, v["out"][n]), n


def test_no_tokens():
    dt, code = DT["bf16"]
    q, k = torch.empty(0, 4, 64, dtype=dt, device="cuda"), torch.empty(0, 2, 64, dtype=dt, device="cuda")
    gamma, dg = torch.ones(64, dtype=dt, device="cuda"), torch.ones(2, 64, dtype=dt, device="cuda")
    dtp.dtp_qk_norm_rotate_forward(0, 4, 2, 64, code, q, k, q, k, gamma_q=gamma, gamma_k=gamma)
    dtp.dtp_qk_norm_rotate_backward(0, 4, 2, 64, code, q, k, q, k, q, k, gamma_q=gamma, gamma_k=gamma, dgamma_q=dg[0],
                                    dgamma_k=dg[1])
    torch.cuda.synchronize()
    assert not bool(dg.any())


def test_not_finite_values_stay_in_their_heads():
    v = run(9, 5, 5, 64, "bf16", packed=False, seed=8)
    q = v["q"].clone()
    q[4, 2, 7] = float("nan")
    out, k_out = torch.empty_like(q), torch.empty_like(v["k"])
    dtp.dtp_qk_norm_rotate_forward(9, 5, 5, 64, dtp.DTP_BF16, q, v["k"], out, k_out, **v["common"])
    torch.cuda.synchronize()
    keep = torch.ones(9, 5, dtype=torch.bool, device="cuda")
    keep[4, 2] = False
    assert bool(torch.isnan(out[4, 2]).all())
    assert torch.equal(out[keep], v["out"]["q"][keep]) and torch.equal(k_out, v["out"]["k"])


def test_gradients_against_differences():
    """fp32: gradients of a weighted sum of outputs against central differences of the forward call
    (a step of 1e-2 leaves errors of 1e-4 in gradients of unit size)."""
    T, H, G, dh = 2, 2, 1, 8
    q, k, cq, ck = normal(1, T, H, dh), normal(2, T, G, dh), normal(3, T, H, dh), normal(4, T, G, dh)
    gq, gk = 1 + normal(5, dh, scale=0.1), 1 + normal(6, dh, scale=0.1)
    pos, inv = torch.tensor([3, 11], dtype=torch.int32, device="cuda"), torch.tensor([1.0, 0.1], device="cuda")
    qo, ko = torch.empty_like(q), torch.empty_like(k)

    def loss(q_, k_, gq_, gk_):
        dtp.dtp_qk_norm_rotate_forward(T, H, G, dh, dtp.DTP_F32, q_, k_, qo, ko, gamma_q=gq_, gamma_k=gk_, positions=pos,
                                       inv_freq=inv)
        return float((qo.double() * cq.double()).sum() + (ko.double() * ck.double()).sum())

    args = (q, k, gq, gk)
    grads = [torch.empty_like(a) for a in args]
    dtp.dtp_qk_norm_rotate_backward(T, H, G, dh, dtp.DTP_F32, q, k, cq, ck, grads[0], grads[1], gamma_q=gq, gamma_k=gk,
                                    positions=pos, inv_freq=inv, dgamma_q=grads[2], dgamma_k=grads[3])
    for i, (a, g) in enumerate(zip(args, grads)):
        for at in range(0, a.numel(), 3):
            v = []
            for e in (1e-2, -1e-2):
                moved = a.clone()
                moved.view(-1)[at] += e
                v.append(loss(*args[:i], moved, *args[i + 1:]))
            assert abs((v[0] - v[1]) / 2e-2 - float(g.view(-1)[at])) < 5e-3, (i, at)


def test_captured_and_replayed_between_eager_calls():
    T, H, G, dh = 300, 8, 4, 128
    dt, code = DT["bf16"]
    sets = [run(T, H, G, dh, "bf16", packed=False, seed=s) for s in (10, 20)]
    common = sets[0]["common"]
    cur = {n: sets[0][n].clone() for n in ("q", "k", "dq_out", "dk_out")}
    ws = workspace(dtp.dtp_qk_norm_rotate_workspace(T, H, G, dh, code))

    def step(i, o, space):
        dtp.dtp_qk_norm_rotate_forward(T, H, G, dh, code, i["q"], i["k"], o["q"], o["k"], **common)
        dtp.dtp_qk_norm_rotate_backward(T, H, G, dh, code, i["q"], i["k"], i["dq_out"], i["dk_out"], o["dq"], o["dk"],
                                        dgamma_q=o["dgq"], dgamma_k=o["dgk"], workspace=space, **common)

    out = {n: torch.empty_like(t) for n, t in sets[0]["out"].items()}
    eager = {n: torch.empty_like(t) for n, t in sets[0]["out"].items()}
    step(cur, out, ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(cur, out, ws)
    for s in (1, 0, 1):
        for n in cur:
            cur[n].copy_(sets[s][n])
        graph.replay()
        step(sets[s], eager, None)
        torch.cuda.synchronize()
        for n in out:
            assert torch.equal(out[n], eager[n]), (s, n)


def test_refusals_on_the_gpu():
    dt, code = DT["bf16"]
    rows = normal(0, 8, 8 * 64, dtype=dt)
    q, k = rows[:, :4 * 64].view(8, 4, 64), rows[:, 4 * 64:6 * 64].view(8, 2, 64)
    g = torch.ones(64, dtype=dt, device="cuda")
    out = torch.empty(8, 4, 64, dtype=dt, device="cuda")
    # an output that starts where a strided input does is not in place
    refused(lambda: dtp.lib() and dtp._check(dtp.lib().dtp_qk_norm_rotate_forward(
        8, 4, 2, 64, code, q.data_ptr(), 512, k.data_ptr(), 512, g.data_ptr(), g.data_ptr(), 1e-6, None, None, 0, q.data_ptr(),
        out.data_ptr(), None)), match="overlaps")
    refused(lambda: dtp.dtp_qk_norm_rotate_forward(8, 4, 2, 64, code, q, k, out, out, gamma_q=g, gamma_k=g), match="overlaps")
    with pytest.raises(ValueError, match="elements"):
        dtp.dtp_qk_norm_rotate_forward(8, 4, 2, 64, code, q, k, out[:4], out, gamma_q=g, gamma_k=g)
    assert GUARD
