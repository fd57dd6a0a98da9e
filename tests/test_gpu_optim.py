"""The gradients' norm and AdamW over many tensors against the formulas.

fp32 steps are compared bit by bit with the same fp32 operations done one after the other on the CPU (IEEE, each rounded),
and with fp64 within what those roundings allow; 8-bit moments with torch's own e4m3 rounding of the fp32 values."""
import math

import pytest
import torch

import paper_2505_07291_amd as grpo

pytestmark = pytest.mark.gpu
BF16, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
SIZES = [1, 3, 255, 256, 257, 1000, 4096, 8191, 8192, 8193, 70001]


def quantise(x, keep=False):
    """(codes, scales) as grpo.h defines them, a block of 256 at a time."""
    n = x.numel()
    x = torch.nn.functional.pad(x, (0, -n % 256)).view(-1, 256)
    top = torch.where(torch.isfinite(x), x, torch.zeros(())).abs().amax(1)
    scales = []
    for t in top.tolist():
        e = -126
        while t > 448.0 * 2.0 ** e:
            e += 1
        scales.append(2.0 ** e)
    scales = torch.tensor(scales, dtype=F32)
    y = x / scales[:, None]
    if keep:
        y = torch.where((x > 0) & (y < 2.0 ** -9), torch.tensor(2.0 ** -9), y)
    y = torch.where(torch.isfinite(y), y, torch.tensor(float("nan")))
    return y.to(E4M3).view(-1)[:n], scales


def root(x):
    """The fp32 square root rounded to nearest: torch's own on the CPU is off by a step for one value in five, while the root
    in fp64 has twice the bits and two more, so that rounding it again gives the nearest."""
    return x.double().sqrt().float()


def cut(sizes, dtype, align):
    """Tensors inside one buffer: align 1 puts them right behind one another, at odd addresses too."""
    starts, at = [], 0
    for n in sizes:
        starts.append(at)
        at += -(-n // align) * align
    buffer = torch.zeros(at + 64, dtype=dtype, device="cuda")
    if dtype == E4M3:
        buffer = buffer.view(torch.uint8)
    off = 0 if align > 1 else 1
    out = [buffer[off + a:off + a + n] for a, n in zip(starts, sizes)]
    return [t.view(E4M3) for t in out] if dtype == E4M3 else out


class Model:
    """Tensors of the given sizes with everything a step needs, and the same on the CPU."""

    def __init__(self, seed, sizes, param="f32", grad=F32, bits=32, align=64, decay=0.01):
        g = torch.Generator().manual_seed(seed)
        rand = lambda n, s: torch.randn(n, generator=g) * s  # noqa: E731
        self.sizes, self.kind, self.bits = sizes, param, bits
        self.decay = [decay * (i % 2) for i in range(len(sizes))]
        pd = F32 if param == "f32" else BF16
        self.params, self.grads = cut(sizes, pd, align), cut(sizes, grad, align)
        self.masters = cut(sizes, F32, align) if param == "master" else None
        sd = F32 if bits == 32 else E4M3
        self.m, self.v = cut(sizes, sd, align), cut(sizes, sd, align)
        self.ms = self.vs = None
        if bits == 8:
            self.ms = [torch.zeros(-(-n // 256), device="cuda") for n in sizes]
            self.vs = [torch.zeros(-(-n // 256), device="cuda") for n in sizes]
        self.host = []
        for i, n in enumerate(sizes):
            p = rand(n, 0.5)
            if param == "bf16":
                p = p.to(BF16).float()
            gr = (rand(n, 1.0) * torch.exp(rand(n, 2.0)) * 10.0 ** (i % 4 - 2)).to(grad)
            m, v = rand(n, 0.1), rand(n, 0.2) ** 2
            h = dict(p=p, g=gr, m=m, v=v)
            if bits == 8:
                h["mq"], h["ms"] = quantise(m)
                h["rq"], h["rs"] = quantise(root(v), keep=True)
            self.host.append(h)
            self.params[i].copy_(p)
            self.grads[i].copy_(gr)
            if self.masters:
                self.masters[i].copy_(p)
            if bits == 8:
                self.m[i].view(torch.uint8).copy_(h["mq"].view(torch.uint8))
                self.v[i].view(torch.uint8).copy_(h["rq"].view(torch.uint8))
                self.ms[i].copy_(h["ms"])
                self.vs[i].copy_(h["rs"])
            else:
                self.m[i].copy_(m)
                self.v[i].copy_(v)
        self.plan = grpo.grpo_optim_plan(self.params, self.grads, self.m, self.v, masters=self.masters, exp_avg_scales=self.ms,
                                         exp_avg_sq_scales=self.vs, weight_decay=self.decay)

    def host_step(self, step, lr, b1, b2, eps, coef=None):
        """The same step on the CPU, every fp32 operation rounded by itself."""
        f = lambda x: torch.tensor(x, dtype=F32)  # noqa: E731
        for h, decay in zip(self.host, self.decay):
            g = h["g"].float()
            g = g * coef if coef is not None else g
            m, v = h["m"], h["v"]
            if self.bits == 8:
                m = h["mq"].float() * h["ms"].repeat_interleave(256)[:m.numel()]
                v = h["rq"].float() * h["rs"].repeat_interleave(256)[:v.numel()]
                v = v * v
            m = m * f(b1) + g * f(1.0 - b1)
            v = v * f(b2) + (g * g) * f(1.0 - b2)
            r = root(v)
            u = m / (r * f(1.0 / math.sqrt(1.0 - b2 ** step)) + f(eps))
            h["p"] = h["p"] * f(1.0 - lr * decay) - u * f(lr / (1.0 - b1 ** step))
            h["out"] = h["p"].to(BF16) if self.kind != "f32" else h["p"]
            if self.kind == "bf16":
                h["p"] = h["out"].float()
            h["m"], h["v"] = m, v
            if self.bits == 8:
                h["mq"], h["ms"] = quantise(m)
                h["rq"], h["rs"] = quantise(r, keep=True)

    def check(self):
        for i, h in enumerate(self.host):
            pairs = dict(param=(self.params[i], h["out"]))
            if self.masters:
                pairs["master"] = (self.masters[i], h["p"])
            if self.bits == 8:
                pairs.update(m=(self.m[i], h["mq"]), v=(self.v[i], h["rq"]), m_scale=(self.ms[i], h["ms"]), v_scale=(self.vs[i], h["rs"]))
            else:
                pairs.update(m=(self.m[i], h["m"]), v=(self.v[i], h["v"]))
            wrong = {k: int((a.cpu().float() != b.float()).sum()) for k, (a, b) in pairs.items()}
            assert not any(wrong.values()), (i, self.sizes[i], wrong)


@pytest.mark.parametrize("align", [64, 1])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad", [F32, BF16])
@pytest.mark.parametrize("param", ["f32", "bf16", "master"])
def test_steps(param, grad, bits, align):
    a = Model(3, SIZES, param, grad, bits, align)
    for step in (1, 2, 3):
        grpo.grpo_adamw_step(a.plan, step, 0.03, 0.9, 0.95, 1e-6)
        a.host_step(step, 0.03, 0.9, 0.95, 1e-6)
        a.check()


def test_against_the_formula_in_64_bits():
    """One step from zero moments: about eight roundings of 2^-24 between gradient and step, two in the parameter."""
    a = Model(5, [5000], "f32")
    a.m[0].zero_()
    a.v[0].zero_()
    p, g = a.params[0].double().cpu(), a.grads[0].double().cpu()
    grpo.grpo_adamw_step(a.plan, 1, 0.1, 0.9, 0.999, 1e-8)
    m, v = 0.1 * g, 0.001 * g * g
    u = 0.1 * (m / (1 - 0.9)) / (torch.sqrt(v / (1 - 0.999)) + 1e-8)
    want = p * (1 - 0.1 * a.decay[0]) - u
    off = (a.params[0].double().cpu() - want).abs()
    # beta in fp32 is off by half a step too, and 1 - beta2 is formed from beta2 in fp64
    assert (off <= 2.0 ** -24 * (2 * p.abs() + 12 * u.abs() + want.abs())).all()


@pytest.mark.parametrize("bits", [8, 32])
def test_offsets_beyond_32_bits(bits):
    """A tensor of more than 2^32 values with gradients at its ends alone: there what tensors of the ends give, zeros between."""
    n, end = 2 ** 32 + 5000, 5000  # (the last 5000 begin with a block of 256)
    g = torch.Generator().manual_seed(bits)
    ends = [torch.randn(end, generator=g).to(BF16).cuda() for _ in range(2)]

    def zeros(n):
        if bits == 8:
            m, v = (torch.zeros(n, dtype=torch.uint8, device="cuda").view(E4M3) for _ in range(2))
            ms, vs = (torch.zeros((n + 255) // 256, device="cuda") for _ in range(2))
        else:
            m, v, ms, vs = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"), None, None
        return dict(p=torch.zeros(n, dtype=BF16, device="cuda"), m=m, v=v, ms=ms, vs=vs)

    def step(states, grads):
        plan = grpo.grpo_optim_plan([t["p"] for t in states], grads, [t["m"] for t in states], [t["v"] for t in states],
                                    exp_avg_scales=[t["ms"] for t in states], exp_avg_sq_scales=[t["vs"] for t in states])
        norm = grpo.grpo_grad_norm(plan, 0.5)
        grpo.grpo_adamw_step(plan, 3, 1e-2, clip=torch.tensor([1.0, 0.25], device="cuda"))
        return norm[0].item()

    big, grad = zeros(n), torch.zeros(n, dtype=BF16, device="cuda")
    grad[:end], grad[n - end:] = ends[0], ends[1]
    small = [zeros(end), zeros(end)]
    assert step([big], [grad]) == pytest.approx(step(small, ends), rel=2.0 ** -23)
    for name in ("p", "m", "v"):
        whole = big[name].view(torch.uint8) if bits == 8 and name != "p" else big[name]
        for part, of in ((whole[:end], small[0]), (whole[n - end:], small[1])):
            assert torch.equal(part, of[name].view(torch.uint8) if bits == 8 and name != "p" else of[name]), name
        for at in range(end, n - end, 2 ** 28):
            assert not whole[at:min(at + 2 ** 28, n - end)].any(), name


def test_one_launch_over_different_tensors():
    """Tensors of every kind in one plan."""
    models = [Model(7 + k, [300, 9000], param, grad, bits, align) for k, (param, grad, bits, align) in
              enumerate([("f32", BF16, 32, 64), ("master", F32, 8, 1), ("bf16", F32, 32, 1), ("f32", F32, 8, 64), ("master", BF16, 32, 64)])]
    join = lambda key: [t for a in models for t in (getattr(a, key) or [None] * 2)]  # noqa: E731
    plan = grpo.grpo_optim_plan(join("params"), join("grads"), join("m"), join("v"), masters=join("masters"), exp_avg_scales=join("ms"),
                                exp_avg_sq_scales=join("vs"), weight_decay=[w for a in models for w in a.decay])
    clip = torch.tensor([3.0, 0.3], device="cuda")
    grpo.grpo_adamw_step(plan, 4, 0.02, clip=clip)
    for a in models:
        a.host_step(4, 0.02, 0.9, 0.999, 1e-8, coef=torch.tensor(0.3))
        a.check()


@pytest.mark.parametrize("align", [64, 1])
@pytest.mark.parametrize("grad", [F32, BF16])
@pytest.mark.parametrize("sizes", [[1], SIZES, [5] * 700, [3000001, 17], [0, 12, 0]])
def test_norm(sizes, grad, align):
    a = cut(sizes, grad, align)
    g = torch.Generator().manual_seed(1)
    for i, t in enumerate(a):
        t.copy_(torch.randn(t.shape, generator=g) * 3.0 ** (i % 3))
    norm = math.sqrt(math.fsum(t.double().square().sum().item() for t in a))
    plan = grpo.grpo_optim_plan(None, a)
    for most in (0.0, norm / 3, norm * 3):
        got = grpo.grpo_grad_norm(plan, most).double().cpu()
        # one rounding to fp32 each; the sums, in fp64, are far inside it
        assert abs(got[0].item() - norm) <= 2.0 ** -24 * norm * 1.0001
        coef = min(1.0, most / norm) if most else 1.0
        assert abs(got[1].item() - coef) <= 2.0 ** -24 * coef * 1.0001
    again = grpo.grpo_grad_norm(plan, norm / 3)
    assert torch.equal(grpo.grpo_grad_norm(plan, norm / 3), again)


def test_norm_of_extremes():
    a = [torch.zeros(1000, device="cuda"), torch.zeros(70000, device="cuda")]
    plan = grpo.grpo_optim_plan(None, a)
    assert grpo.grpo_grad_norm(plan, 0.1).tolist() == [0.0, 1.0]
    a[1].fill_(1e30)  # squares beyond fp32
    assert abs(grpo.grpo_grad_norm(plan, 1.0)[0].item() / (1e30 * math.sqrt(70000)) - 1) < 1e-6
    a[0][7] = float("inf")
    assert grpo.grpo_grad_norm(plan, 1.0).tolist() == [float("inf"), 0.0]
    a[0][8] = float("nan")
    assert all(math.isnan(x) for x in grpo.grpo_grad_norm(plan, 1.0).tolist())


@pytest.mark.parametrize("bits", [32, 8])
def test_what_is_not_finite_stays_where_it_is(bits):
    a = Model(9, [1000, 600], "master", F32, bits)
    a.grads[0][10], a.grads[0][700], a.grads[1][3] = float("nan"), float("inf"), float("-inf")
    for i, j in ((0, 10), (0, 700), (1, 3)):
        a.host[i]["g"] = a.grads[i].cpu()
    grpo.grpo_adamw_step(a.plan, 1, 0.01)
    a.host_step(1, 0.01, 0.9, 0.999, 1e-8)
    for i, h in enumerate(a.host):
        for got, want in ((a.params[i], h["out"]), (a.masters[i], h["p"])):
            got = got.cpu()
            bad = ~torch.isfinite(want)
            assert torch.equal(bad, ~torch.isfinite(got)) and torch.equal(got[~bad], want[~bad]) and bad.sum() == (2, 1)[i]
        if bits == 8:
            for got, want, sg, sw in ((a.m[i], h["mq"], a.ms[i], h["ms"]), (a.v[i], h["rq"], a.vs[i], h["rs"])):
                got, want = got.cpu().float(), want.float()
                assert torch.equal(got.isnan(), want.isnan()) and want.isnan().sum() == (2, 1)[i]
                assert torch.equal(got.nan_to_num(), want.nan_to_num()) and torch.equal(sg.cpu(), sw)


def test_every_e4m3_value_and_border():
    """Codes for values on, and next to, every border between e4m3 values: one block whose largest value makes the scale 1."""
    values = torch.arange(256, dtype=torch.uint8).view(E4M3).float()
    values = values[torch.isfinite(values) & (values >= 0)].sort().values
    mid = (values[1:].double() + values[:-1].double()) / 2
    x = torch.cat([values.double(), mid, mid * (1 - 2 ** -20), mid * (1 + 2 ** -20)]).float()
    blocks = [torch.cat([torch.tensor([448.0]), b]) for b in x.split(255)]
    x = torch.cat([torch.nn.functional.pad(b, (0, 256 - b.numel())) for b in blocks])
    n = x.numel()
    # beta1 = 0 and a gradient of x: m becomes x; moments, parameters and their scales of nothing
    for sign in (1.0, -1.0):
        one = dict(device="cuda")
        p, g = torch.zeros(n, **one), (sign * x).cuda()
        m, v = (torch.zeros(n, dtype=torch.uint8, **one).view(E4M3) for _ in range(2))
        ms, vs = (torch.zeros(n // 256, **one) for _ in range(2))
        plan = grpo.grpo_optim_plan([p], [g], [m], [v], exp_avg_scales=[ms], exp_avg_sq_scales=[vs])
        grpo.grpo_adamw_step(plan, 1, 0.0, 0.0, 0.0, 0.0)
        assert (ms == 1.0).all() and (vs == 1.0).all()
        assert torch.equal(m.cpu().float(), (sign * x).to(E4M3).float())
        r = root(x.square())
        want = torch.where((r > 0) & (r < 2.0 ** -9), torch.tensor(2.0 ** -9), r).to(E4M3).float()
        assert torch.equal(v.cpu().float(), want)


def test_second_moments_do_not_vanish():
    """A value whose second moment is far below its block's: without a least code the next step would be m / eps."""
    g = torch.full((256,), 1e-7, device="cuda")
    g[0] = 1e3
    p = torch.zeros(256, device="cuda")
    m, v = (torch.zeros(256, dtype=torch.uint8, device="cuda").view(E4M3) for _ in range(2))
    ms, vs = (torch.zeros(1, device="cuda") for _ in range(2))
    plan = grpo.grpo_optim_plan([p], [g], [m], [v], exp_avg_scales=[ms], exp_avg_sq_scales=[vs])
    for step in range(1, 6):
        grpo.grpo_adamw_step(plan, step, 1.0, eps=1e-12)
        assert (v.float() > 0).all() and p.abs().max() <= 1.01 * step


def test_clip_and_step_replayed():
    """norm, clip and step in a graph, the step's number and the learning rate on the device: every replay is an eager step."""
    a, b = (Model(11, SIZES, "master", F32, 8) for _ in range(2))
    step, lr = torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(1, device="cuda")

    def call():
        step.add_(1)
        clip = grpo.grpo_grad_norm(a.plan, 0.1)
        grpo.grpo_adamw_step(a.plan, step, lr, clip=clip)
        return clip

    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        clip = call()
    for k in range(1, 6):
        for t, u in zip(a.grads, b.grads):
            t.mul_(0.5 + k)
            u.copy_(t)
        lr.fill_(2.0 ** -k)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = grpo.grpo_grad_norm(b.plan, 0.1)
        grpo.grpo_adamw_step(b.plan, k, 2.0 ** -k, clip=want)
        assert torch.equal(clip, want)
        # the corrections 1 - beta^k come from expm1 there and from pow here: half a step of fp32, and what follows from it
        for s, t in zip(a.masters, b.masters):
            assert (s - t).abs().max() <= 2.0 ** -20 * 2.0 ** -k * 4 + 2.0 ** -22 * t.abs().max()


def test_on_another_stream():
    a, b = (Model(13, SIZES, "master", BF16, 32) for _ in range(2))
    stream = torch.cuda.Stream()
    out, ws = torch.zeros(2, device="cuda"), torch.zeros(1 << 15, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    grpo.grpo_grad_norm(a.plan, 0.1, norm_out=out, workspace=ws, stream=stream)
    grpo.grpo_adamw_step(a.plan, 1, 0.1, clip=out, stream=stream)
    stream.synchronize()
    grpo.grpo_adamw_step(b.plan, 1, 0.1, clip=grpo.grpo_grad_norm(b.plan, 0.1))
    for s, t in zip(a.masters + a.m, b.masters + b.m):
        assert torch.equal(s, t)
