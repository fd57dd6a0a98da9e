"""The new operators' calls from Python: the binding's native part gives the bits of the general path, and whatever is not a call
that grpo.h allows is refused, with nothing written."""
import pytest
import torch

import paper_2505_07291_amd as grpo
from paper_2505_07291_amd import binding

pytestmark = pytest.mark.gpu
BF16, F32, F64, I32, I64 = torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.int64


def rnd(*shape, dtype=BF16):
    return torch.randn(shape, device="cuda").to(dtype)


def verify_args(n=5, k=3, v=264, dtype=BF16):
    return dict(target_logits=rnd(n, k + 1, v, dtype=dtype), draft_logits=rnd(n, k, v, dtype=dtype),
                draft_tokens=torch.randint(0, v, (n, k), device="cuda"), accept_u=torch.rand((n, k), device="cuda"),
                sample_u=torch.rand(n, device="cuda", dtype=F64), draft_lengths=torch.randint(-1, k + 1, (n,), device="cuda", dtype=I32))


def norm_args(n=7, d=264, dtype=BF16):
    return dict(residual=rnd(n, d), block=rnd(n, d, dtype=dtype), post_weight=rnd(d), gate=rnd(n, d), pre_weight=rnd(d))


def bits(out):
    return [t.clone().view(torch.uint8) if t is not None else None for t in out]


class General:
    """The general path."""

    def __enter__(self):
        self.fast, binding._fast = binding._fast, binding._NoFastcall()

    def __exit__(self, *a):
        binding._fast = self.fast


def both(call):
    taken = call()
    with General():
        general = call()
    for a, b in zip(bits(taken), bits(general)):
        assert (a is None) == (b is None) and (a is None or torch.equal(a, b))
    for a, b in zip(taken, general):
        assert a is None or (a.shape == b.shape and a.stride() == b.stride() and a.dtype == b.dtype)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_native_part_and_general_path_agree(dtype):
    grpo.lib()
    a = verify_args(dtype=dtype)
    both(lambda: grpo.grpo_verify_drafts(**a, temperature=0.7, draft_temperature=2))
    both(lambda: grpo.grpo_verify_drafts(**dict(a, draft_logits=None, draft_lengths=None)))
    both(lambda: grpo.grpo_verify_drafts(a["target_logits"][:, :1], None, None, None, a["sample_u"]))
    both(lambda: grpo.grpo_verify_drafts(**{k: v[:1] for k, v in a.items()}))
    for n, d in ((7, 264), (1, 5), (3, 5121)):
        g = norm_args(n, d + (8 - d % 8) % 8)
        g = {k: t[..., :d] if t.dim() == 2 else t[:d] for k, t in g.items()}
        dh, dx = rnd(n, d + (8 - d % 8) % 8)[:, :d], rnd(n, d + (8 - d % 8) % 8)[:, :d]
        back = {k: v for k, v in g.items() if k != "residual"}
        for drop in ((), ("gate",), ("post_weight",), ("pre_weight",), ("block", "gate", "post_weight")):
            f, b = dict(g, **{k: None for k in drop}), dict(back, **{k: None for k in drop})
            both(lambda: grpo.grpo_block_norm_fwd(**f, residual_scale=0.5))
            both(lambda: grpo.grpo_block_norm_bwd(g["residual"], **b, grad_hidden=None if "pre_weight" in drop else dh, grad_residual_out=dx))
        both(lambda: grpo.grpo_block_norm_fwd(**dict(g, gate=g["gate"][0].contiguous())))
        both(lambda: grpo.grpo_block_norm_bwd(g["residual"], **dict(back, gate=g["gate"][0].contiguous()), grad_hidden=dh))
    p = [rnd(1000, dtype=dtype), rnd(7, dtype=dtype)]
    m, v = [torch.zeros(1000, device="cuda"), torch.zeros(7, device="cuda")], [torch.zeros(1000, device="cuda"), torch.zeros(7, device="cuda")]
    grads = [rnd(1000, dtype=F32), rnd(7, dtype=F32)]
    plan = grpo.grpo_optim_plan(p, grads, m, v)
    both(lambda: [grpo.grpo_grad_norm(plan, 0.5)])

    def step():
        for t, s in zip(p + m + v, start):
            t.copy_(s)
        grpo.grpo_adamw_step(plan, 3, 1e-2, clip=grpo.grpo_grad_norm(plan, 0.5))
        return [t.clone() for t in p + m + v]

    start = [t.clone() for t in p + m + v]
    both(step)


def refused(match, f, *a, error=ValueError, **k):
    with pytest.raises(error, match=match):
        f(*a, **k)


def test_verify_refusals():
    a = verify_args()
    f = grpo.grpo_verify_drafts
    for change, match in [
            (dict(target_logits=a["target_logits"].half()), "target_logits"), (dict(target_logits=a["target_logits"][0]), "target_logits"),
            (dict(target_logits=a["target_logits"].transpose(1, 2).contiguous().transpose(1, 2)), "unit stride"),
            (dict(draft_logits=a["draft_logits"].float()), "draft_logits"), (dict(draft_logits=a["draft_logits"][:, :2]), "draft_logits"),
            (dict(draft_logits=a["draft_logits"].cpu()), "live on"), (dict(draft_tokens=a["draft_tokens"].int()), "draft_tokens"),
            (dict(draft_tokens=a["draft_tokens"][:, :2]), "draft_tokens"), (dict(draft_tokens=None), "draft_tokens"),
            (dict(accept_u=a["accept_u"].double()), "accept_u"), (dict(accept_u=None), "accept_u"),
            (dict(sample_u=a["sample_u"].float()), "sample_u"), (dict(sample_u=a["sample_u"][:2]), "sample_u"),
            (dict(draft_lengths=a["draft_lengths"].long()), "draft_lengths"), (dict(draft_lengths=a["draft_lengths"][:1]), "draft_lengths")]:
        refused(match, f, **dict(a, **change))
    out = torch.full((5, 4), 7, dtype=I64, device="cuda")
    refused("PARAM|parameter", f, **a, temperature=0.0, tokens_out=out, error=grpo.GrpoError)
    refused("aligned", f, **dict(a, target_logits=rnd(5, 4, 265)[:, :, 1:]), error=grpo.GrpoError)
    refused("workspace", f, **a, tokens_out=out, workspace=torch.zeros(256, dtype=torch.uint8, device="cuda"), error=grpo.GrpoError)
    refused("tokens_out", f, **a, tokens_out=out[:, :3])
    assert (out == 7).all()
    refused("shape", f, rnd(2, 66, 8), rnd(2, 65, 8), torch.zeros((2, 65), dtype=I64, device="cuda"), torch.zeros((2, 65), device="cuda"),
            a["sample_u"][:2], error=grpo.GrpoError)


def test_block_norm_refusals():
    a = norm_args()
    for change, match in [
            (dict(residual=a["residual"].double()), "residual"), (dict(residual=a["residual"][0]), "residual"),
            (dict(residual=a["residual"].t().contiguous().t()), "unit stride"), (dict(block=a["block"][:3]), "block"),
            (dict(block=a["block"].half()), "float32 or bfloat16"), (dict(block=a["block"].cpu()), "live on"),
            (dict(post_weight=a["post_weight"].float()), "post_weight"), (dict(post_weight=a["post_weight"][:8]), "post_weight"),
            (dict(gate=a["gate"][:, :8]), "gate"), (dict(gate=a["gate"][:1].expand(7, -1)), "gate"),
            (dict(pre_weight=a["pre_weight"].float()), "pre_weight"), (dict(pre_weight=None, hidden=rnd(7, 264)), "hidden"),
            (dict(hidden=rnd(7, 264, dtype=F32)), "hidden"), (dict(residual_out=rnd(6, 264)), "residual_out"),
            (dict(block=None, post_weight=None, gate=None, residual_out=rnd(7, 264)), "residual_out")]:
        refused(match, grpo.grpo_block_norm_fwd, **dict(a, **change))
    refused("NULL", grpo.grpo_block_norm_fwd, a["residual"], None, a["post_weight"], pre_weight=a["pre_weight"], error=grpo.GrpoError)
    refused("NULL", grpo.grpo_block_norm_fwd, a["residual"], error=grpo.GrpoError)
    refused("aligned", grpo.grpo_block_norm_fwd, **dict(a, residual=rnd(7, 265)[:, 1:]), error=grpo.GrpoError)
    refused("dtype", grpo.grpo_block_norm_fwd, a["residual"], a["block"].float(), error=grpo.GrpoError)
    refused("parameter", grpo.grpo_block_norm_fwd, **a, eps=-1.0, error=grpo.GrpoError)
    back = dict(residual_out=a["residual"], block=a["block"], post_weight=a["post_weight"], gate=a["gate"], pre_weight=a["pre_weight"],
                grad_hidden=rnd(7, 264))
    for change, match in [(dict(grad_hidden=None), "grad_hidden"), (dict(pre_weight=None), "grad_hidden"),
                          (dict(grad_hidden=rnd(7, 264, dtype=F32)), "grad_hidden"), (dict(grad_residual_out=rnd(7, 264, dtype=F32)), "grad_residual_out"),
                          (dict(grad_residual=rnd(7, 200)), "grad_residual"), (dict(grad_block=rnd(7, 264, dtype=F32)), "grad_block"),
                          (dict(grad_gate=rnd(264, dtype=F32)), "grad_gate"), (dict(grad_post_weight=rnd(264)), "grad_post_weight"),
                          (dict(accumulate_grad_weights=True), "needs")]:
        refused(match, grpo.grpo_block_norm_bwd, **dict(back, **change))
    refused("workspace", grpo.grpo_block_norm_bwd, **back, workspace=torch.zeros(256, dtype=torch.uint8, device="cuda"), error=grpo.GrpoError)


def test_optimiser_refusals():
    p, g, m, v = ([rnd(300, dtype=F32), rnd(20, dtype=F32)] for _ in range(4))
    f = grpo.grpo_optim_plan
    e = [torch.zeros(n, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for n in (300, 20)]
    s = [torch.zeros(n, device="cuda") for n in (2, 1)]
    for a, k, match in [
            ((p, g[:1], m, v), {}, "params"), ((p, g, m[:1], v), {}, "exp_avgs"), ((p, g, m, v), dict(weight_decay=[0.1]), "weight_decay"),
            (([p[0].double(), p[1]], g, m, v), {}, "params"), ((p, [g[0].half(), g[1]], m, v), {}, "grads"),
            (([p[0][:200], p[1]], g, m, v), {}, "param has"), ((p, g, m, [v[0][:10], v[1]]), {}, "exp_avg_sq has"),
            ((p, g, [rnd(600, dtype=F32)[::2], m[1]], v), {}, "contiguous"), ((p, g, m, [v[0].cpu(), v[1]]), {}, "exp_avg_sqs"),
            ((p, g, m, [e[0], v[1]]), {}, "same dtype"), ((p, g, e, [t.clone() for t in e]), dict(exp_avg_scales=[s[0][:1], s[1]]), "every 256")]:
        refused(match, f, *a, **k)
    refused("memory", f, p, g, m, [m[0], v[1]], error=grpo.GrpoError)          # the same moments twice
    refused("memory", f, p, [p[0], g[1]], m, v, error=grpo.GrpoError)          # a gradient that is the parameter
    refused("memory", f, [p[0], p[0][10:30]], g, m, v, error=grpo.GrpoError)   # a tensor inside another
    refused("NULL", f, p, g, e, [t.clone() for t in e], error=grpo.GrpoError)  # 8 bits without scales
    refused("NULL", f, p, g, m, v, exp_avg_scales=s, exp_avg_sq_scales=[t.clone() for t in s], error=grpo.GrpoError)
    refused("dtype", f, p, g, m, v, masters=[rnd(300, dtype=F32), rnd(20, dtype=F32)], error=grpo.GrpoError)
    plan = f(p, g, m, v)
    refused("parameter", grpo.grpo_adamw_step, plan, 0, 0.1, error=grpo.GrpoError)
    refused("parameter", grpo.grpo_adamw_step, plan, 1, 0.1, 1.0, error=grpo.GrpoError)
    refused("step", grpo.grpo_adamw_step, plan, torch.ones(1, device="cuda"), 0.1)
    refused("lr", grpo.grpo_adamw_step, plan, 1, torch.ones(2, device="cuda"))
    refused("clip", grpo.grpo_adamw_step, plan, 1, 0.1, clip=torch.ones(1, device="cuda"))
    refused("NULL", grpo.grpo_adamw_step, f(None, g), 1, 0.1, error=grpo.GrpoError)
    refused("norm_out", grpo.grpo_grad_norm, plan, norm_out=torch.zeros(1, device="cuda"))
    refused("parameter", grpo.grpo_grad_norm, plan, float("nan"), error=grpo.GrpoError)
