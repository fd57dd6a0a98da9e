"""The norms around a block and their gradients against the formulas in fp64.

Tolerances: what is written in bf16 is off by half a step, 2^-8 of the value (fp32: 2^-24).  Before that, fp32 sums of up to
20000 terms, each lane's share in order (at most 80 terms) and lanes pairwise, and some ten operations after them: under
128 * 2^-24 of the sum of the operands' magnitudes, which the references below give beside each value.  Sums over rows
add at most 80 rows in order in fp32: 256 * 2^-24 of the terms' magnitudes."""
import pytest
import torch

import paper_2505_07291_amd as grpo

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
STEP = {BF16: 2.0 ** -8, F32: 2.0 ** -24}
U = 128 * 2.0 ** -24


def rows(g, n, d, dtype, scale=1.0, shift=0.0, pad=0):
    per16 = 8 if dtype == BF16 else 4
    pitch = (d + per16 - 1) // per16 * per16 + pad * per16
    t = torch.full((max(n, 1), pitch), 777.0, dtype=dtype)
    t[:n, :d] = (torch.randn((n, d), generator=g) * scale + shift).to(dtype)
    return t.cuda()[:n, :d]


def make(seed, n, d, res=BF16, dt=BF16, block=True, post=True, gate="full", pre=True, pad=0):
    g = torch.Generator().manual_seed(seed)
    s = dict(residual=rows(g, n, d, res, 3.0, pad=pad))
    s["block"] = rows(g, n, d, dt, 1.5, pad=pad) if block else None
    s["post_weight"] = rows(g, 1, d, dt, 0.2, 1.0)[0].contiguous() if post else None
    s["pre_weight"] = rows(g, 1, d, dt, 0.2, 1.0)[0].contiguous() if pre else None
    s["gate"] = {"none": None, "full": rows(g, n, d, dt, pad=pad), "row": rows(g, 1, d, dt)[0].contiguous()}[gate]
    return s, dict(grad_hidden=rows(g, n, d, dt, 0.1, pad=pad) if pre else None, grad_residual_out=rows(g, n, d, res, 0.1, pad=pad))


def wide(s):
    return {k: None if v is None else v.double().cpu() for k, v in s.items()}


def inv_rms(x, eps):
    return 1.0 / torch.sqrt((x * x).mean(1, keepdim=True) + eps)


def forward(s, scale, eps):
    """((x', magnitude), (h, magnitude))"""
    x, f = s["residual"], s["block"]
    size = x.abs()
    if f is not None:
        b = f if s["post_weight"] is None else f * inv_rms(f, eps) * s["post_weight"]
        b = b if s["gate"] is None else b * s["gate"]
        x, size = x + scale * b, size + (scale * b).abs()
    if s["pre_weight"] is None:
        return (x, size), None
    r = inv_rms(x, eps)
    return (x, size), (x * r * s["pre_weight"], size * r * s["pre_weight"].abs())


def backward(s, grads, scale, eps):
    x, f = s["residual"], s["block"]
    out = {}
    dxo = grads["grad_residual_out"]
    D = torch.zeros_like(x) if dxo is None else dxo
    size = D.abs()
    if s["pre_weight"] is not None:
        r = inv_rms(x, eps)
        y, a = x * r, s["pre_weight"] * grads["grad_hidden"]
        D = D + r * (a - y * (a * y).mean(1, keepdim=True))
        size = size + r * (a.abs() + y.abs() * (a * y).abs().mean(1, keepdim=True))
        out["grad_pre_weight"] = ((grads["grad_hidden"] * y).sum(0), 2 * (grads["grad_hidden"] * y).abs().sum(0))
    out["grad_residual"] = (D, size)
    if f is None:
        return out
    r = 1.0 if s["post_weight"] is None else inv_rms(f, eps)
    y = f * r
    w = 1.0 if s["post_weight"] is None else s["post_weight"]
    g = 1.0 if s["gate"] is None else s["gate"]
    sD, sS = scale * D, abs(scale) * size
    wa, ga = (v.abs() if isinstance(v, torch.Tensor) else v for v in (w, g))
    t, ts = sD * g * w, sS * ga * wa
    if s["post_weight"] is None:
        out["grad_block"] = (t, ts)
    else:
        out["grad_block"] = (r * (t - y * (t * y).mean(1, keepdim=True)), r * (ts + y.abs() * (ts * y.abs()).mean(1, keepdim=True)))
        out["grad_post_weight"] = ((sD * g * y).sum(0), 2 * (sS * ga * y.abs()).sum(0))
    if s["gate"] is not None:
        gg, gs = sD * w * y, sS * wa * y.abs()
        out["grad_gate"] = (gg, gs) if s["gate"].dim() == 2 else (gg.sum(0), 2 * gs.sum(0))
    return out


def near(got, want, what):
    value, size = want
    g = got.double().cpu()
    off = (g - value).abs()
    allowed = STEP[got.dtype] * (value.abs() + U * size) + U * size + 1e-37
    worst = (off / allowed).max().item() if off.numel() else 0.0
    assert torch.isfinite(g).all() and worst <= 1.0, (what, worst)


NAMES = ("grad_residual", "grad_block", "grad_gate", "grad_post_weight", "grad_pre_weight")


def check(s, grads, scale=0.5, eps=1e-6):
    x, h = grpo.grpo_block_norm_fwd(**s, residual_scale=scale, eps=eps)
    want = forward(wide(s), scale, eps)
    near(x, want[0], "residual_out")
    assert (h is None) == (want[1] is None)
    if h is not None:
        near(h, want[1], "hidden")
    back = {k: v for k, v in s.items() if k != "residual"}
    got = dict(zip(NAMES, grpo.grpo_block_norm_bwd(s["residual"], **back, **grads, residual_scale=scale, eps=eps)))
    want = backward(wide(s), wide(grads), scale, eps)
    assert {k for k, v in got.items() if v is not None} == set(want)
    for k, v in want.items():
        near(got[k], v, k)


@pytest.mark.parametrize("res,dt", [(BF16, BF16), (F32, BF16), (F32, F32)])
@pytest.mark.parametrize("n,d", [(1, 1), (3, 3), (3, 7), (2, 8), (2, 64), (5, 255), (130, 257), (7, 768), (33, 1000), (2, 2048), (3, 2049), (9, 4104),
                                 (1, 5120), (70, 5120), (600, 5123),
                                 (4, 8192), (2, 8200), (3, 9001), (5, 10240), (300, 10243), (2, 16384), (3, 16391), (2, 19456), (1, 20001)])
def test_sizes(n, d, res, dt):
    check(*make(n * 100003 + d, n, d, res, dt))


@pytest.mark.parametrize("res,dt", [(BF16, BF16), (F32, BF16), (F32, F32)])
@pytest.mark.parametrize("n,d", [(37, 520), (19, 5120), (3, 17000)])
@pytest.mark.parametrize("block,post,gate,pre", [(True, True, "full", True), (True, True, "row", True), (True, True, "none", True),
                                                 (True, False, "full", True), (True, False, "row", True), (True, False, "none", True),
                                                 (True, True, "full", False), (True, True, "row", False), (True, False, "row", False),
                                                 (True, False, "none", False), (False, False, "none", True)])
def test_parts_that_are_left_out(n, d, res, dt, block, post, gate, pre):
    s, grads = make(7, n, d, res, dt, block, post, gate, pre)
    check(s, grads, scale=-0.75)
    if pre:  # nothing but the norm has a gradient
        check(s, dict(grads, grad_residual_out=None))


def test_pitches_and_what_lies_between_rows():
    for res, dt in ((BF16, BF16), (F32, BF16)):
        s, grads = make(3, 21, 523, res, dt, pad=3)
        check(s, grads)
        out = {k: torch.full((21, 560), 5.0, dtype=t, device="cuda") for k, t in
               (("residual_out", res), ("hidden", dt), ("grad_residual", res), ("grad_block", dt), ("grad_gate", dt))}
        cut = {k: v[:, :523] for k, v in out.items()}
        grpo.grpo_block_norm_fwd(**s, residual_out=cut["residual_out"], hidden=cut["hidden"])
        back = {k: v for k, v in s.items() if k != "residual"}
        grpo.grpo_block_norm_bwd(s["residual"], **back, **grads, **{k: v for k, v in cut.items() if k.startswith("grad")})
        for k, v in out.items():
            assert (v[:, 523:] == 5.0).all() and torch.isfinite(v).all(), k


@pytest.mark.parametrize("n", [0, 1, 255, 256, 257, 1023, 1025, 3001, 9000])
def test_sums_over_rows(n):
    """More rows than workgroups, and none at all."""
    s, grads = make(n, n, 136, gate="row")
    if n:
        check(s, grads)
    back = {k: v for k, v in s.items() if k != "residual"}
    first = grpo.grpo_block_norm_bwd(s["residual"], **back, **grads)
    again = grpo.grpo_block_norm_bwd(s["residual"], **back, **grads)
    for a, b in zip(first, again):
        assert torch.equal(a, b)
    # the gradients of two micro-batches add up
    more = [t.clone() for t in first[2:]]
    grpo.grpo_block_norm_bwd(s["residual"], **back, **grads, grad_gate=more[0], grad_post_weight=more[1], grad_pre_weight=more[2],
                             accumulate_grad_weights=True)
    for a, b in zip(first[2:], more):
        assert torch.equal(a + a, b)
    if n == 0:
        assert all(not t.any() for t in first[2:])


def test_offsets_beyond_32_bits():
    """Rows that lie 3 GB apart: what the same rows close together give, bit for bit."""
    s, grads = make(11, 3, 520)
    far = 1500000000 // 8 * 8

    def apart(t):
        big = torch.empty(2 * far + 520, dtype=BF16, device="cuda").as_strided((3, 520), (far, 1))
        return big if t is None else big.copy_(t)

    close = grpo.grpo_block_norm_fwd(**s)
    moved = {k: apart(v) if torch.is_tensor(v) and v.dim() == 2 else v for k, v in s.items()}
    out = dict(residual_out=apart(None), hidden=apart(None))
    grpo.grpo_block_norm_fwd(**moved, **out)
    assert torch.equal(out["residual_out"], close[0]) and torch.equal(out["hidden"], close[1])
    back = {k: v for k, v in s.items() if k != "residual"}
    close = grpo.grpo_block_norm_bwd(s["residual"], **back, **grads)
    back = {k: v for k, v in moved.items() if k != "residual"}
    far_grads = {k: apart(v) for k, v in grads.items()}
    out = dict(grad_residual=apart(None), grad_block=apart(None), grad_gate=apart(None))
    got = grpo.grpo_block_norm_bwd(moved["residual"], **back, **far_grads, **out)
    for a, b in zip(got, close):
        assert torch.equal(a, b)


def test_in_place():
    for res, d in ((BF16, 776), (F32, 776), (F32, 20000)):
        s, grads = make(5, 40, d, res)
        x, h = grpo.grpo_block_norm_fwd(**s)
        copy = s["residual"].clone()
        x2, h2 = grpo.grpo_block_norm_fwd(**dict(s, residual=copy), inplace=True)
        assert x2 is copy and torch.equal(x, x2) and torch.equal(h, h2)
        back = {k: v for k, v in s.items() if k != "residual"}
        a = grpo.grpo_block_norm_bwd(x, **back, **grads)
        copy = grads["grad_residual_out"].clone()
        b = grpo.grpo_block_norm_bwd(x, **back, **dict(grads, grad_residual_out=copy), grad_residual=copy)
        assert b[0] is copy and all(torch.equal(u, v) for u, v in zip(a, b))


def test_gradients_are_those_of_differences():
    """The backward against central differences of the forward's formula: the two agree with one another, not only with
    formulas derived the same way."""
    s, grads = make(11, 3, 24, F32, F32, gate="row")
    names = ("block", "gate", "post_weight", "pre_weight")
    w = wide(s)
    g = wide(grads)
    x_in = w["residual"]

    def value(t):
        (x, _), (h, _) = forward(t, 0.5, 1e-6)
        return (x * g["grad_residual_out"]).sum() + (h * g["grad_hidden"]).sum()

    x_out = forward(w, 0.5, 1e-6)[0][0].float().cuda()
    back = {k: v for k, v in s.items() if k != "residual"}
    got = dict(zip(("residual",) + names, grpo.grpo_block_norm_bwd(x_out, **back, **grads, residual_scale=0.5)))
    for name in ("residual",) + names:
        base = w[name].clone()
        flat = base.view(-1)
        for i in range(0, flat.numel(), 5):
            d = []
            for h in (1e-5, -1e-5):
                t = flat.clone()
                t[i] += h
                d.append(value(dict(w, **{name: t.view(base.shape)})))
            slope = ((d[0] - d[1]) / 2e-5).item()
            assert abs(got[name].view(-1)[i].item() - slope) <= 1e-5 * max(1.0, abs(slope)), (name, i)
    assert x_in is w["residual"]


def test_zero_rows_infinities_and_nan_stay_in_their_rows():
    s, grads = make(2, 6, 512)
    s["residual"][1] = 0
    s["block"][1] = 0
    s["block"][3, 5] = float("inf")
    s["residual"][4, 500] = float("nan")
    x, h = grpo.grpo_block_norm_fwd(**s)
    assert not x[1].any() and not h[1].any()
    back = {k: v for k, v in s.items() if k != "residual"}
    dx, df, dg, _, _ = grpo.grpo_block_norm_bwd(x, **back, **grads)
    for t in (x, h, dx, df, dg):
        fine = torch.isfinite(t).all(1).tolist()
        assert fine[0] and fine[1] and fine[2] and fine[5] and not fine[3] and not fine[4]


@pytest.mark.parametrize("n,d", [(1, 5120), (300, 768)])
def test_captured_and_replayed(n, d):
    s, grads = make(1, n, d, gate="row")
    back = {k: v for k, v in s.items() if k != "residual"}

    def step():
        x, h = grpo.grpo_block_norm_fwd(**s)
        return (x, h) + grpo.grpo_block_norm_bwd(x, **back, **grads)

    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        out = step()
    for k in range(4):
        s["block"].mul_(1.25)
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out)), k


def test_on_another_stream():
    s, _ = make(1, 64, 1024)
    want = grpo.grpo_block_norm_fwd(**s)
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    out = [torch.zeros_like(t) for t in want]
    torch.cuda.synchronize()
    grpo.grpo_block_norm_fwd(**s, residual_out=out[0], hidden=out[1], stream=stream)
    stream.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, out))
