"""The operators together, as a rollout and an optimiser step use them: drafted tokens are verified, their tokens and log-probs go
to the objective, the block's norms stand in front of the head, and all weights' gradients are clipped and applied."""
import math

import numpy as np
import pytest
import torch

import paper_2505_07291_amd as grpo
from test_gpu_verify import reference

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
B, K, V, D = 12, 3, 520, 128
EPS = 1e-6
CLIP = dict(eps_low=0.2, eps_high=0.2, delta=4.0)


def policy(seed):
    g = torch.Generator().manual_seed(seed)
    rand = lambda *s, scale=1.0, shift=0.0: (torch.randn(s, generator=g) * scale + shift).to(BF16).cuda()  # noqa: E731
    n = B * (K + 1)
    return dict(residual=rand(n, D, scale=2.0), block=rand(n, D), gate=rand(D, scale=0.5), post=rand(D, scale=0.1, shift=1.0),
                pre=rand(D, scale=0.1, shift=1.0), weight=rand(V, D, scale=0.25)), g


def rollout(s, g):
    """Tokens, log-probs and mask of B responses of up to K + 1 tokens, from drafts that a noisy copy of the policy made."""
    _, hidden = grpo.grpo_block_norm_fwd(s["residual"], s["block"], s["post"], s["gate"], s["pre"], residual_scale=0.5, eps=EPS)
    logits = (hidden.float() @ s["weight"].float().t()).to(BF16).view(B, K + 1, V)
    draft = (logits[:, :K].float().cpu() + 0.5 * torch.randn((B, K, V), generator=g)).to(BF16).cuda()
    drafted = torch.multinomial(torch.softmax(draft.float().cpu(), -1).view(-1, V), 1, generator=g).view(B, K)
    u, v = torch.rand((B, K), generator=g), torch.rand(B, generator=g, dtype=torch.float64)
    tokens, accepted, logprobs = grpo.grpo_verify_drafts(logits, draft, drafted.cuda(), u.cuda(), v.cuda())
    want = reference(logits, draft, drafted, u, v, None)
    assert np.array_equal(tokens.cpu().numpy(), want[0]) and np.array_equal(accepted.cpu().numpy(), want[1])
    mask = (torch.arange(K + 1, device="cuda") <= accepted[:, None]).to(torch.uint8).view(-1)
    return tokens.view(-1), logprobs.view(-1), mask


def gradients(s, tokens, old, adv, mask, denom, into=None):
    x, hidden = grpo.grpo_block_norm_fwd(s["residual"], s["block"], s["post"], s["gate"], s["pre"], residual_scale=0.5, eps=EPS)
    more = {} if into is None else dict(grad_weight=into[0], accumulate_grad_weight=True)
    loss, _, _, dh, dw = grpo.grpo_lmhead_loss_fwd_bwd(hidden, s["weight"], tokens, old, adv, mask, denom=denom, **CLIP, **more)
    more = {} if into is None else dict(grad_gate=into[1], grad_post_weight=into[2], grad_pre_weight=into[3], accumulate_grad_weights=True)
    dx, df, dg, dpost, dpre = grpo.grpo_block_norm_bwd(x, s["block"], s["post"], s["gate"], s["pre"], dh, residual_scale=0.5, eps=EPS, **more)
    return loss, [dw, dg, dpost, dpre], dx, df


def by_autograd(s, tokens, old, adv, mask, denom):
    w = {k: v.double().cpu().requires_grad_() for k, v in s.items()}
    norm = lambda t: t / torch.sqrt(t.square().mean(1, keepdim=True) + EPS)  # noqa: E731
    x = w["residual"] + 0.5 * w["gate"] * norm(w["block"]) * w["post"]
    z = (norm(x) * w["pre"]) @ w["weight"].t()
    m = mask.cpu().bool()
    lp = torch.log_softmax(z, -1)[m].gather(1, tokens.cpu()[m][:, None])[:, 0]
    r, a = torch.exp(lp - old.cpu().double()[m]), adv.cpu().double()[m]
    j = torch.minimum(torch.minimum(r, torch.tensor(CLIP["delta"])) * a, r.clamp(1 - CLIP["eps_low"], 1 + CLIP["eps_high"]) * a)
    loss = -j.sum() / denom
    names = ["weight", "gate", "post", "pre", "residual", "block"]
    return loss.item(), dict(zip(names, torch.autograd.grad(loss, [w[k] for k in names])))


def test_rollout_and_step():
    s, g = policy(1)
    tokens, old, mask = rollout(s, g)
    live = int(mask.sum())
    adv = torch.randn(B, generator=g).repeat_interleave(K + 1).cuda()
    # the rollout is a little old: some tokens are clipped, some not
    old = (old + 0.1 * torch.randn(old.shape, generator=g).cuda()) * mask
    names = ["weight", "gate", "post", "pre"]
    loss, grads, dx, df = gradients(s, tokens, old, adv, mask, live)
    want_loss, want = by_autograd(s, tokens, old, adv, mask, live)
    # three roundings to bf16 lie behind one another (hidden states, logits' gradient, hidden states' gradient), and one of what is
    # written: 2^-8 each, of terms whose signs vary, so that 2-norms are off by about as much; the loss by the first alone
    assert abs(loss.item() - want_loss) <= 2.0 ** -8 * adv.abs().max().item()
    for got, name in zip(grads + [dx, df], names + ["residual", "block"]):
        off = (got.double().cpu() - want[name]).norm() / want[name].norm()
        assert off <= 4 * 2.0 ** -8, (name, off)

    # two micro-batches, half of the responses each, add up to the same gradients: fp32 sums in another order, and the same bf16 terms
    halves = [mask.clone(), mask.clone()]
    halves[0][B // 2 * (K + 1):] = 0
    halves[1][:B // 2 * (K + 1)] = 0
    total = [torch.zeros_like(t) for t in grads]
    for h in halves:
        gradients(s, tokens, old, adv, h, live, into=total)
    for a, b, name in zip(grads, total, names):
        assert (a - b).norm() <= 2.0 ** -16 * a.norm(), name

    # clipped and applied, moments in 8 bits for the head and in 32 for the vectors
    params = [s[k] for k in names]
    masters = [t.float() for t in params]
    before = [t.double().cpu() for t in masters]
    e4m3 = lambda t: torch.zeros(t.numel(), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)  # noqa: E731
    zeros = lambda t: torch.zeros(t.numel(), device="cuda")  # noqa: E731
    scales = [torch.zeros(V * D // 256, device="cuda") if i == 0 else None for i in range(4)]
    more = [torch.zeros(V * D // 256, device="cuda") if i == 0 else None for i in range(4)]
    plan = grpo.grpo_optim_plan(params, grads, [e4m3(t) if i == 0 else zeros(t) for i, t in enumerate(params)],
                                [e4m3(t) if i == 0 else zeros(t) for i, t in enumerate(params)], masters=masters, exp_avg_scales=scales,
                                exp_avg_sq_scales=more, weight_decay=[0.1, 0.0, 0.0, 0.0])
    norm = math.sqrt(sum(t.double().square().sum().item() for t in grads))
    clip = grpo.grpo_grad_norm(plan, norm / 4)
    assert abs(clip[0].item() / norm - 1) <= 2.0 ** -23 and abs(clip[1].item() - 0.25) <= 2.0 ** -24
    grpo.grpo_adamw_step(plan, 1, 1e-3, 0.9, 0.999, 1e-12, clip=clip)
    for p, m, old_p, gr, decay in zip(params, masters, before, grads, (0.1, 0.0, 0.0, 0.0)):
        # the first step is lr * g / |g|, but for eps; ten fp32 roundings of a step and two of the parameter
        step = 1e-3 * torch.sign(gr.double().cpu())
        step = step * (gr.double().cpu().abs() > 1e-9)
        off = (m.double().cpu() - (old_p * (1 - 1e-3 * decay) - step)).abs()
        assert (off <= 1e-3 * (16 * 2.0 ** -24 + 1e-12 / (0.25 * 1e-9)) + 3 * 2.0 ** -24 * old_p.abs())[gr.cpu().abs() > 1e-9].all()
        assert torch.equal(p, m.to(BF16))
    # the next rollout is the new policy's
    rollout(s, g)
