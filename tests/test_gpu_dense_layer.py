"""The dense operators run together, as a decoder layer uses them: the whole forward pass around an
attention, the same layer after its layout is applied, shards' partial sums, the operating point
that the affinity scores see, a training step of the FFN, and sizes whose offsets pass 32 bits."""
import math
import sys

import pytest
import torch

from paper_2609_13846_amd import dtp
from tests import dense_reference as ref
from tests.test_gpu_dense import DT, normal, workspace

pytestmark = pytest.mark.gpu

EPS = 1e-6


def announce(*a):
    print("[gpu]", *a, file=sys.stderr, flush=True)


def weights(d, I, H, G, dh, dt, seed=0):
    shapes = dict(w_q=(H * dh, d), w_k=(G * dh, d), w_v=(G * dh, d), w_o=(d, H * dh), w_gate=(I, d), w_up=(I, d),
                  w_down=(d, I))
    w = {k: normal(seed + i, *s, scale=s[1] ** -0.5, dtype=dt) for i, (k, s) in enumerate(shapes.items())}
    for i, k in enumerate(("g_attn", "g_ffn")):
        w[k] = (1 + normal(seed + 20 + i, d, scale=0.1)).to(dt)
    for i, k in enumerate(("g_q", "g_k")):
        w[k] = (1 + normal(seed + 30 + i, dh, scale=0.1)).to(dt)
    return w


def rms(x, gain):
    x = x.double()
    return x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * gain.double()


def attention(q, k, v):
    """Causal attention of [T, H, dh] with G key heads, in 64 bits."""
    T, H, dh = q.shape
    q, k, v = q.double(), k.double(), v.double()
    k, v = (t.repeat_interleave(H // t.shape[1], 1).transpose(0, 1).contiguous() for t in (k, v))
    s = torch.bmm(q.transpose(0, 1).contiguous(), k.transpose(1, 2).contiguous()) / math.sqrt(dh)
    s = s.masked_fill(torch.ones(T, T, dtype=torch.bool, device=s.device).triu(1), -math.inf)
    return torch.bmm(s.softmax(-1), v).transpose(0, 1)


def positions(T):
    return torch.arange(T, dtype=torch.int32, device="cuda") + 5000


def frequencies(dh):
    return (1e4 ** (-torch.arange(dh // 2, dtype=torch.float64) * 2 / dh)).float().cuda()


def run_layer(x0, w, H, G, dh, dtype):
    """x0 -> (x, attn, x_next) by the operators; norms and attention are torch's, rounded to the type."""
    dt, code = DT[dtype]
    T, d = x0.shape
    I, width = w["w_gate"].shape[0], (H + 2 * G) * dh

    def buffer(*shape):
        return torch.empty(*shape, dtype=dt, device="cuda")

    qkv, q, k = buffer(T, width), buffer(T, H, dh), buffer(T, G, dh)
    w_qkv = torch.cat((w["w_q"], w["w_k"], w["w_v"]))
    dtp.dtp_linear_forward(T, d, width, code, rms(x0, w["g_attn"]).to(dt), w_qkv, qkv)
    dtp.dtp_qk_norm_rotate_forward(T, H, G, dh, code, qkv[:, :H * dh].view(T, H, dh),
                                   qkv[:, H * dh:(H + G) * dh].view(T, G, dh), q, k, gamma_q=w["g_q"], gamma_k=w["g_k"],
                                   eps=EPS, positions=positions(T), inv_freq=frequencies(dh))
    attn = attention(q, k, qkv[:, (H + G) * dh:].view(T, G, dh)).to(dt).contiguous()
    x, h, x_next = buffer(T, d), buffer(T, I), buffer(T, d)
    dtp.dtp_linear_forward(T, H * dh, d, code, attn.view(T, H * dh), w["w_o"], x, residual=x0)
    dtp.dtp_gated_forward(T, d, I, code, rms(x, w["g_ffn"]).to(dt), w["w_gate"], w["w_up"], h)
    dtp.dtp_linear_forward(T, I, d, code, h, w["w_down"], x_next, residual=x)
    torch.cuda.synchronize()
    return x, attn, x_next, h


def layer_64(x0, w, H, G, dh):
    T = x0.shape[0]
    w = {k: v.double() for k, v in w.items()}
    n = rms(x0, w["g_attn"])
    q, k = (n @ w["w_q"].t()).view(T, H, dh), (n @ w["w_k"].t()).view(T, G, dh)
    q, k = (ref.turn(rms(t, g), positions(T), frequencies(dh)) for t, g in ((q, w["g_q"]), (k, w["g_k"])))
    x = x0.double() + attention(q, k, (n @ w["w_v"].t()).view(T, G, dh)).reshape(T, H * dh) @ w["w_o"].t()
    n = rms(x, w["g_ffn"])
    h = torch.nn.functional.silu(n @ w["w_gate"].t()) * (n @ w["w_up"].t())
    return x, x + h @ w["w_down"].t()


def rel(a, b):
    return float((a.double() - b.double()).norm() / b.double().norm())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,I,H,G,dh", [(1, 256, 640, 8, 4, 32), (37, 200, 333, 6, 2, 40), (150, 512, 1024, 8, 2, 64)])
def test_layer_forward(dtype, T, d, I, H, G, dh):
    """Eight roundings to the type between x0 and x_next, each at most u of the value it is of: 8 u in
    norm where every step passes errors on as it does values (in fp32 the sums' own roundings,
    at most I 2^-23, are more)."""
    announce("layer", dtype, T, d, I, H, G, dh)
    dt, _ = DT[dtype]
    w = weights(d, I, H, G, dh, dt)
    x0 = normal(99, T, d, dtype=dt)
    x, _, x_next, _ = run_layer(x0, w, H, G, dh, dtype)
    want_x, want_next = layer_64(x0, w, H, G, dh)
    bar = 8 * ref.U[dt] + (I * 2.0 ** -23 if dtype == "f32" else 0)
    assert rel(x, want_x) < bar and rel(x_next, want_next) < bar


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("L", [2, 4])
def test_layer_after_its_layout_is_applied(dtype, L):
    """The permuted layer is the same function: what differs is the order of the sums over heads and
    neurons, so two runs are no further apart than each from the exact one."""
    T, d, I, H, G, dh = 60, 256, 512, 8, 4, 32
    dt, code = DT[dtype]
    w = weights(d, I, H, G, dh, dt)
    h, nu = dtp.dtp_random_layout(1, G, I, L, 7)
    moved = {k: torch.empty_like(w[k]) for k in dtp.WEIGHT_ORDER}
    dtp.dtp_apply_layout(d, I, H, G, dh, code, L, h[0], nu[0], {k: w[k] for k in dtp.WEIGHT_ORDER}, moved)
    x0 = normal(98, T, d, dtype=dt)
    a, b = run_layer(x0, w, H, G, dh, dtype), run_layer(x0, {**w, **moved}, H, G, dh, dtype)
    bar = 2 * (8 * ref.U[dt] + (I * 2.0 ** -23 if dtype == "f32" else 0))
    assert rel(b[0], a[0]) < bar and rel(b[2], a[2]) < bar
    _, order = dtp.dtp_layout_orders(G, I, L, h[0], nu[0])
    if dtype == "f32":  # every neuron's value, where the layout put it
        assert rel(b[3], a[3][:, torch.from_numpy(order).long().cuda()]) < bar


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_shards_add_up_to_the_layer(dtype):
    """Each device's neurons through their columns of W_down, added onto the residual in turn, in place:
    the dense block, to a rounding per device."""
    T, d, I, L = 45, 192, 512, 4
    dt, code = DT[dtype]
    w = weights(d, I, 4, 2, 32, dt)
    x = normal(1, T, d, dtype=dt)
    n = rms(x, w["g_ffn"]).to(dt)
    y, h = x.clone(), torch.empty(T, I // L, dtype=dt, device="cuda")
    for s in range(L):
        at = slice(s * I // L, (s + 1) * I // L)
        dtp.dtp_gated_forward(T, d, I // L, code, n, w["w_gate"][at], w["w_up"][at], h)
        dtp.dtp_linear_forward(T, I // L, d, code, h, w["w_down"][:, at].contiguous(), y, residual=y)
    whole, hw = torch.empty_like(y), torch.empty(T, I, dtype=dt, device="cuda")
    dtp.dtp_gated_forward(T, d, I, code, n, w["w_gate"], w["w_up"], hw)
    dtp.dtp_linear_forward(T, I, d, code, hw, w["w_down"], whole, residual=x)
    torch.cuda.synchronize()
    assert rel(y, whole) < (L + 1) * ref.U[dt] + I * 2.0 ** -23


def test_operating_point_of_the_affinity_scores():
    """s_down of the affinity pass, sum_t alpha_k^2 / r'^2, is that of the gated block's h (fp32).  Each
    side's g and u are off by at most the sums' roundings, and three more for the gain and 1/r
    on the affinity's side: twice the block's own bound and four steps per factor."""
    T, d, I, H, G, dh = 200, 128, 320, 4, 2, 32
    w = weights(d, I, H, G, dh, torch.float32, seed=3)
    x0 = normal(97, T, d)
    x, attn, x_next, _ = run_layer(x0, w, H, G, dh, "f32")
    layer = dtp.dtp_layer_create(d, I, H, G, dh, EPS, dtp.DTP_F32)
    try:
        dtp.dtp_layer_set_weights(layer, w["w_o"], w["g_ffn"], w["w_gate"], w["w_up"], w["w_down"])
        A, s = torch.zeros(G, I, device="cuda"), torch.zeros(I, device="cuda")
        dtp.dtp_affinity_accumulate_down(layer, x, attn, x_next, EPS, T, A, s)
        torch.cuda.synchronize()
    finally:
        dtp.dtp_layer_destroy(layer)
    n = rms(x, w["g_ffn"]).float()
    h = torch.empty(T, I, device="cuda")
    dtp.dtp_gated_forward(T, d, I, dtp.DTP_F32, n, w["w_gate"], w["w_up"], h)
    _, eh, _ = ref.gated(n, w["w_gate"], w["w_up"])
    e = 3 * eh + 16 * 2.0 ** -24 * (n.double().abs() @ w["w_gate"].double().abs().t()) * \
        (1 + (n.double().abs() @ w["w_up"].double().abs().t()))
    r2 = (x_next.double() ** 2).mean(-1, keepdim=True) + EPS
    want = (h.double() ** 2 / r2).sum(0)
    bound = ((2 * h.double().abs() * e + e * e) / r2).sum(0) + ref.summed(T) * want
    ref.check(s, want, bound, "s_down")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,d,I", [(1, 96, 200), (90, 130, 301), (300, 256, 640)])
def test_training_step_of_the_ffn(dtype, T, d, I):
    """y = x + sqrt(2) h W_down, h the gated block of x: all gradients through both backward calls.  Four
    roundings to the type (h, dh, dg and du, the result) stand between dy and a gradient."""
    dt, code = DT[dtype]
    announce("ffn step", dtype, T, d, I)
    x, dy = normal(1, T, d, dtype=dt), normal(2, T, d, dtype=dt)
    wg, wu = (normal(s, I, d, scale=d ** -0.5, dtype=dt) for s in (3, 4))
    wd = normal(5, d, I, scale=I ** -0.5, dtype=dt)
    alpha = math.sqrt(2.0)
    space = workspace(max(dtp.dtp_gated_workspace(T, d, I, code, True), dtp.dtp_linear_workspace(T, I, d, code, backward=True)))
    h, y = torch.empty(T, I, dtype=dt, device="cuda"), torch.empty(T, d, dtype=dt, device="cuda")
    pre = torch.empty(T, 2, I, device="cuda")
    dh, dx = torch.empty_like(h), torch.empty_like(x)
    dwg, dwu, dwd = torch.empty_like(wg), torch.empty_like(wu), torch.empty_like(wd)
    dtp.dtp_gated_forward(T, d, I, code, x, wg, wu, h, pre=pre, workspace=space)
    dtp.dtp_linear_forward(T, I, d, code, h, wd, y, residual=x, alpha=alpha, workspace=space)
    dtp.dtp_linear_backward(T, I, d, code, h, wd, dy, dx=dh, dw=dwd, alpha=alpha, workspace=space)
    dtp.dtp_gated_backward(T, d, I, code, x, wg, wu, pre, dh, dx=dx, dw_gate=dwg, dw_up=dwu, workspace=space)
    torch.cuda.synchronize()
    leaves = [t.double().requires_grad_() for t in (x, wg, wu, wd)]
    xx, gg, uu, dd = leaves
    out = xx + alpha * (torch.nn.functional.silu(xx @ gg.t()) * (xx @ uu.t())) @ dd.t()
    want = torch.autograd.grad(out, leaves, dy.double())
    bar = 4 * ref.U[dt] + (max(I, T) * 2.0 ** -23 if dtype == "f32" else 0)
    assert rel(y, out.detach()) < bar
    for name, got, v in (("dx", dx.double() + dy.double(), want[0]), ("dw_gate", dwg, want[1]), ("dw_up", dwu, want[2]),
                         ("dw_down", dwd, want[3])):
        assert rel(got, v) < bar, name


@pytest.mark.parametrize("dtype,T,N", [("bf16", 290000, 8192), ("f32", 150000, 16384)])
def test_offsets_beyond_32_bits(dtype, T, N):
    """More than 2^31 outputs: the last tokens' results are those of a call on them alone, and the
    weights' gradient over all tokens is the formula's on some rows."""
    K = 32
    dt, code = DT[dtype]
    announce("far offsets", dtype, T, N)
    assert T * N > 2 ** 31
    x, w = normal(1, T, K, dtype=dt), normal(2, N, K, scale=0.2, dtype=dt)
    y = torch.empty(T, N, dtype=dt, device="cuda")
    dtp.dtp_linear_forward(T, K, N, code, x, w, y)
    last = slice(T - 300, T)
    part = torch.empty(300, N, dtype=dt, device="cuda")
    dtp.dtp_linear_forward(300, K, N, code, x[last].clone(), w, part)
    value, bound, _, _ = ref.linear(x[last], w)
    ref.check(y[last], value, bound, "y")
    ref.check(part, value, bound, "part")
    dx, dw = torch.empty_like(x), torch.empty_like(w)
    dtp.dtp_linear_backward(T, K, N, code, x, w, y, dx=dx, dw=dw)
    some = torch.tensor([0, 1, N // 2, N - 1], device="cuda")
    grads = ref.linear_grads(x[last], w, y[last])
    ref.check(dx[last], *grads["dx"], "dx")
    cols = y[:, some].contiguous()
    grads = ref.linear_grads(x, w[some], cols)
    ref.check(dw[some], *grads["dw"], "dw")


def test_far_offsets_of_heads():
    T, H, G, dh = 530000, 32, 1, 128
    dt, code = DT["bf16"]
    announce("far offsets of heads")
    q, k = normal(1, T, H, dh, dtype=dt), normal(2, T, G, dh, dtype=dt)
    g, pos = torch.ones(dh, dtype=dt, device="cuda"), torch.arange(T, dtype=torch.int32, device="cuda")
    assert q.numel() > 2 ** 31
    last = slice(T - 100, T)
    want, bound = ref.qk(q[last], g, EPS, pos[last], frequencies(dh))
    dout = q[last].clone()
    grads = ref.qk_grads(q[last], g, EPS, pos[last], frequencies(dh), dout)
    dq, dk = torch.empty_like(q), torch.empty_like(k)
    dtp.dtp_qk_norm_rotate_backward(T, H, G, dh, code, q, k, q, k, dq, dk, gamma_q=g, gamma_k=g, eps=EPS, positions=pos,
                                    inv_freq=frequencies(dh))
    ref.check(dq[last], *grads["d"], "dq")
    del dq
    dtp.dtp_qk_norm_rotate_forward(T, H, G, dh, code, q, k, q, k, gamma_q=g, gamma_k=g, eps=EPS, positions=pos,
                                   inv_freq=frequencies(dh))
    ref.check(q[last], want, bound, "q")


def test_more_tokens_than_a_launch_of_small_tiles_takes():
    """2^29 fp32 tokens and some: 64 a tile and 512 threads would be 2^32 threads and more."""
    T = 2 ** 29 + 70
    announce("many tokens", T)
    x = torch.arange(T, dtype=torch.int32, device="cuda").remainder_(1009).float()
    w, y = torch.full((1, 1), 0.5, device="cuda"), torch.full((T,), -1.0, device="cuda")
    space = workspace(dtp.dtp_linear_workspace(T, 1, 1, dtp.DTP_F32))
    dtp.dtp_linear_forward(T, 1, 1, dtp.DTP_F32, x, w, y, workspace=space)
    assert torch.equal(y, x.mul_(0.5))  # exact: halves of whole numbers
    dtp.dtp_linear_backward(T, 1, 1, dtp.DTP_F32, None, w, y, dx=x)
    assert torch.equal(x, y.mul_(0.5))
