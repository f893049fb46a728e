"""The large tiles of the dense operators' products (tests/dense_tiles.py lists the sizes, and
tests/test_dense_plan.py holds the launches to them).

Small whole numbers make every sum exact in 32 bits, in any order, so that results are compared bit for
bit: no term may be missing, doubled or in another row, however long the contraction.  Gradients of
the gated block get pre-activations of 0 and 128, where silu is 0 and 128 and its derivative 1/2
and 1 exactly.  The activations' own values are compared with their formulas in 64 bits, element by
element (tests/dense_reference.py derives the bounds)."""
import sys

import pytest
import torch

from paper_2609_13846_amd import dtp
from tests import dense_reference as ref
from tests.dense_tiles import CASES
from tests.test_gpu_dense import ACT, DT, Out, check_gated, check_linear, normal, run_gated, run_linear, workspace

pytestmark = pytest.mark.gpu


def announce(*a):
    print("[gpu]", *a, file=sys.stderr, flush=True)


def whole(seed, most, *shape):
    """Whole numbers from -most to most, fp32."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-most, most + 1, shape, generator=g, device="cuda").float()


def ids(c):
    return "-".join(map(str, c[:5]))


def product(a, b):
    """a b^T of whole numbers, exact."""
    return a.double() @ b.double().t()


LINEAR, GATED = ([c for c in CASES if c[0] == kind] for kind in ("linear", "gated"))


@pytest.mark.parametrize("case", LINEAR, ids=ids)
def test_linear_sums_are_whole(case):
    _, dtype, T, K, N, _ = case
    announce("linear", *case[:5])
    dt, code = DT[dtype]
    x, w, dy = whole(1, 2, T, K).to(dt), whole(2, 2, N, K).to(dt), whole(3, 2, T, N).to(dt)
    b, r = whole(4, 8, N).to(dt), whole(5, 8, T, N).to(dt)
    assert 2 * (4 * max(T, K, N) + 8) + 8 < 2 ** 24
    space = workspace(dtp.dtp_linear_workspace(T, K, N, code, backward=True))
    y, pre = Out(T, N, dtype=dt), Out(T, N, dtype=torch.float32)
    dtp.dtp_linear_forward(T, K, N, code, x, w, y.t, bias=b, residual=r, alpha=2.0, pre=pre.t, workspace=space)
    z = product(x, w) + b.double()
    assert torch.equal(pre.t.double(), z)
    assert torch.equal(y.t, (r.double() + 2 * z).to(dt))
    in_place = Out(T, N, dtype=dt)
    in_place.t.copy_(r)
    dtp.dtp_linear_forward(T, K, N, code, x, w, in_place.t, bias=b, residual=in_place.t, alpha=2.0, workspace=space)
    assert torch.equal(in_place.t, y.t)
    plain = Out(T, N, dtype=dt)
    dtp.dtp_linear_forward(T, K, N, code, x, w, plain.t, workspace=space)
    assert torch.equal(plain.t, (z - b.double()).to(dt))
    dx, dw, db = Out(T, K, dtype=dt), Out(N, K, dtype=dt), Out(N, dtype=dt)
    dtp.dtp_linear_backward(T, K, N, code, x, w, dy, dx=dx.t, dw=dw.t, dbias=db.t, alpha=2.0, workspace=space)
    assert torch.equal(dx.t, (2 * product(dy, w.t())).to(dt))
    assert torch.equal(dw.t, (2 * product(dy.t(), x.t())).to(dt))
    assert torch.equal(db.t, (2 * dy.double().sum(0)).to(dt))
    assert all(o.untouched() for o in (y, pre, in_place, plain, dx, dw, db))


@pytest.mark.parametrize("case", GATED, ids=ids)
def test_gated_sums_are_whole(case):
    _, dtype, T, d, I, _ = case
    announce("gated", *case[:5])
    dt, code = DT[dtype]
    x, wg, wu = whole(1, 2, T, d).to(dt), (whole(2, 2, I, d) / 64).to(dt), (whole(3, 2, I, d) / 64).to(dt)
    space = workspace(dtp.dtp_gated_workspace(T, d, I, code, True))
    h, pre, alone = Out(T, I, dtype=dt), Out(T, 2, I, dtype=torch.float32), Out(T, I, dtype=dt)
    dtp.dtp_gated_forward(T, d, I, code, x, wg, wu, h.t, pre=pre.t, workspace=space)
    dtp.dtp_gated_forward(T, d, I, code, x, wg, wu, alone.t, workspace=space)
    g, u = product(x, wg), product(x, wu)
    assert torch.equal(pre.t[:, 0].double(), g) and torch.equal(pre.t[:, 1].double(), u)
    want = ref.act(g, "silu")[0] * u
    # g and u are exact: the activation's error, a product, a rounding
    e = (ref.ACT[dt] * g.abs() + 2.0 ** -22 * ref.act(g, "silu")[0].abs()) * u.abs()
    ref.check(h.t, want, e + ref.U[dt] * (want.abs() + e), "h")
    assert torch.equal(alone.t, h.t)
    del want, e, g, u
    # dg = dh u / 2 and du = 0, or dg = dh u and du = 128 dh
    gate, up, dh = 128.0 * (whole(4, 1, T, I) > 0), whole(5, 2, T, I), 2 * whole(6, 1, T, I)
    assert (128 * 2 * 2 + 4 * 2) * max(T, I) < 2 ** 24
    pre.t[:, 0], pre.t[:, 1] = gate, up
    dg = (dh * up * torch.where(gate > 0, 1.0, 0.5)).to(dt)
    du = (dh * gate).to(dt)
    dx, dwg, dwu = Out(T, d, dtype=dt), Out(I, d, dtype=dt), Out(I, d, dtype=dt)
    dtp.dtp_gated_backward(T, d, I, code, x, wg, wu, pre.t, dh.to(dt), dx=dx.t, dw_gate=dwg.t, dw_up=dwu.t, workspace=space)
    assert torch.equal(dx.t, (product(dg, wg.t()) + product(du, wu.t())).to(dt))
    assert torch.equal(dwg.t, product(dg.t(), x.t()).to(dt))
    assert torch.equal(dwu.t, product(du.t(), x.t()).to(dt))
    assert all(o.untouched() for o in (h, pre, alone, dx, dwg, dwu))


# Of each forward tile, with rows that end in whole pieces and not: activation, bias, residual, kept
# pre-activations, and the gradients through them.
ACTIVE = [c for c in CASES if c[2:5] in {(16739, 776, 1200), (15155, 192, 1589), (17232, 192, 392), (17904, 208, 402),
                                         (2624, 520, 6904), (2160, 1347, 80), (3520, 192, 3488), (10320, 792, 975),
                                         (18816, 192, 200), (14208, 208, 258), (16606, 192, 1368), (5512, 104, 181)}]


@pytest.mark.parametrize("case", ACTIVE, ids=ids)
def test_activations(case):
    kind, dtype, T, K, N, _ = case
    assert len(ACTIVE) == 12
    act = "gelu" if N % 3 else "silu"
    announce(*case[:5], act)
    if kind == "linear":
        check_linear(run_linear(T, K, N, dtype, act, -0.75, seed=T), act, -0.75)
    else:
        check_gated(run_gated(T, K, N, dtype, act, seed=T), act)


@pytest.mark.parametrize("case", [c for c in CASES if c[2:5] in {(2054, 808, 4824), (16739, 776, 1200)}], ids=ids)
def test_not_finite_values_stay_in_their_rows(case):
    """Of tiles whose items follow each other: a token's NaN reaches that token's results alone."""
    kind, dtype, T, K, N, _ = case
    dt, code = DT[dtype]
    x, w, wu = normal(1, T, K, dtype=dt), normal(2, N, K, scale=K ** -0.5, dtype=dt), normal(3, N, K, scale=K ** -0.5, dtype=dt)
    bad, at = x.clone(), (0, 255, 256, T // 2, T - 1)
    for i, t in enumerate(at):
        bad[t, (i * 97) % K] = float("nan")
    bad[T - 1, K - 1] = float("inf")
    y = [torch.empty(T, N, dtype=dt, device="cuda") for _ in range(2)]
    for out, v in zip(y, (x, bad)):
        if kind == "linear":
            dtp.dtp_linear_forward(T, K, N, code, v, w, out, act=ACT["gelu"])
        else:
            dtp.dtp_gated_forward(T, K, N, code, v, w, wu, out)
    keep = torch.ones(T, dtype=torch.bool, device="cuda")
    keep[list(at)] = False
    assert torch.equal(y[0][keep], y[1][keep])
    assert bool(torch.isnan(y[1][list(at)]).all())
