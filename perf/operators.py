"""Timed cases of the operators around the objective: what produces its tokens, what stands in front of the language-model
head, and what is done with the gradients.

``path`` names the operator:

  verify    drafted tokens against the target's probabilities: accepted drafts, one more token, their log-probs
  norm_fwd  a block's output normed, gated, scaled and added to the residual stream, and the sum normed for what follows
  norm_bwd  the gradients of all of it
  clip      the norm of all gradients, and the coefficient that clips it
  adamw     one AdamW step over many tensors, moments in 32 bits or in 8

Each has a plain form of elementary torch operations (``own`` false) and the library's call (``own`` true) on the same
inputs.  Vocabularies, widths and option values are those of the package's workloads, tests and benchmark.
"""
import math

import torch

own = False  # whether run() calls the library

DEV = "cuda:0"
EPS = 1e-6
RESIDUAL_SCALE = 0.5
MAX_NORM = 0.1
BETA1, BETA2, ADAM_EPS, LR, STEP, DECAY = 0.9, 0.95, 1e-8, 1e-5, 100, 0.01
QUANT = 256  # values to a scale of the 8-bit moments
TINY_CODE = 2.0 ** -9  # the smallest positive e4m3 value


def listed():
    return [
        # one token each for a few running responses, nothing drafted: what a decoding loop calls for every token
        dict(name="verify_token", path="verify", batch=4, drafts=0, vocab=152064, dtype="bf16", draft="logits", temperature=1.0),
        # one response, four drafted tokens: latency
        dict(name="verify_single", path="verify", batch=1, drafts=4, vocab=152064, dtype="bf16", draft="logits", temperature=1.0),
        # fp32 logits of a vocabulary that is not padded, tokens drafted from the text itself (no draft model)
        dict(name="verify_ragged", path="verify", batch=24, drafts=3, vocab=50257, dtype="f32", draft="tokens", temperature=0.7),
        # a rollout worker's whole batch
        dict(name="verify_batch", path="verify", batch=96, drafts=5, vocab=152064, dtype="bf16", draft="logits", temperature=1.0),
        # one token on its way through a 32B-sized model
        dict(name="norm_token", path="norm_fwd", rows=1, d_model=5120, dtype="bf16", residual="bf16", gate="full", post=True),
        # a training batch in front of the head ...
        dict(name="norm_rows", path="norm_fwd", rows=16384, d_model=5120, dtype="bf16", residual="f32", gate="full", post=True),
        # ... and its gradients
        dict(name="norm_grad", path="norm_bwd", rows=16384, d_model=5120, dtype="bf16", residual="f32", gate="full", post=True),
        # a small model's micro-batch with one learned gate for all rows, whose gradient is a sum over them
        dict(name="norm_grad_small", path="norm_bwd", rows=1000, d_model=768, dtype="bf16", residual="bf16", gate="row", post=True),
        # the gradients of a small model
        dict(name="clip_small", path="clip", vocab=0, d_model=768, layers=2, grad="f32", pad=256),
        # the small model: many tensors of very different sizes, moments in 8 bits
        dict(name="adamw_8bit", path="adamw", vocab=50304, d_model=768, layers=12, grad="bf16", param="master", bits=8, pad=256),
        # the head of a 32B-sized model, as the head's backward leaves its gradient
        dict(name="clip_head", path="clip", vocab=152064, d_model=5120, layers=0, grad="f32", pad=256),
        dict(name="adamw_head", path="adamw", vocab=152064, d_model=5120, layers=0, grad="f32", param="master", bits=32, pad=256),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges, sizes from a logarithmic spread."""
    path = rng.choice(["verify", "verify", "norm_fwd", "norm_bwd", "clip", "adamw"])
    if path == "verify":
        case = dict(path=path, vocab=_log_int(rng, 1000, 300000), drafts=rng.choice([0, 1, 2, 3, 4, 5, 6, 8]),
                    dtype=rng.choice(["bf16", "bf16", "f32"]), draft=rng.choice(["logits", "logits", "tokens"]),
                    temperature=rng.choice([0.7, 1.0, 1.3]))
        if rng.random() < 0.6:  # most trainers pad the vocabulary
            case["vocab"] -= case["vocab"] % 64
        most = 96 * 11 * 152064 * 2 // ((2 * case["drafts"] + 1) * case["vocab"] * _bytes(case["dtype"]))
        case["batch"] = min(_log_int(rng, 1, 256), max(1, most))
        return case
    if path.startswith("norm"):
        dtype = rng.choice(["bf16", "bf16", "f32"])
        case = dict(path=path, d_model=_log_int(rng, 64, 16384), dtype=dtype, residual="f32" if dtype == "f32" else rng.choice(["bf16", "f32"]),
                    gate=rng.choice(["full", "row", "none"]), post=rng.random() < 0.8)
        if rng.random() < 0.8:
            case["d_model"] -= case["d_model"] % 64
        case["rows"] = min(_log_int(rng, 1, 32768), 16384 * 5120 * 2 // (case["d_model"] * _bytes(dtype)))
        return case
    case = dict(path=path, vocab=rng.choice([0, _log_int(rng, 1000, 152064)]), d_model=_log_int(rng, 64, 2048), layers=rng.randrange(1, 25),
                grad=rng.choice(["f32", "bf16"]))
    case["layers"] = min(case["layers"], max(1, (1 << 28) // (12 * case["d_model"] ** 2)))
    if path == "adamw":
        case.update(param=rng.choice(["f32", "bf16", "master"]), bits=rng.choice([8, 32]))
    # tensors of their own begin anywhere in their storage's pages; those cut out of one long buffer, at any value
    case["pad"] = rng.choice([256, 1]) if case.get("bits", 32) == 32 else 256
    return case


def _bytes(dtype):
    return 4 if dtype == "f32" else 2


def _dtype(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _rows(g, n, width, dtype, scale, shift=0.0):
    """[n, width] of normal values whose rows begin on 16-byte boundaries."""
    per16 = 16 // _bytes(dtype)
    pitch = (width + per16 - 1) // per16 * per16
    t = torch.zeros((n, pitch), dtype=_dtype(dtype), device=DEV)[:, :width]
    t.copy_(torch.randn((n, width), generator=g, device=DEV).mul_(scale).add_(shift))
    return t


def _prepare_verify(case, g):
    n, k, v = case["batch"], case["drafts"], case["vocab"]
    per16 = 16 // _bytes(case["dtype"])
    pitch = (v + per16 - 1) // per16 * per16
    z = torch.randn((n, k + 1, v), generator=g, device=DEV).mul_(3.0)
    # a few likely continuations each, as a language model has them
    liked = torch.randint(0, v, (n, k + 1, 8), generator=g, device=DEV)
    z.scatter_add_(2, liked, torch.rand((n, k + 1, 8), generator=g, device=DEV).mul_(6.0).add_(6.0))
    target = torch.zeros((n, k + 1, pitch), dtype=_dtype(case["dtype"]), device=DEV)[:, :, :v]
    target.copy_(z)
    # the draft model's logits are near the target's, and its tokens come from them
    q = z[:, :k] + torch.randn((n, k, v), generator=g, device=DEV).mul_(0.6)
    del z
    draft = torch.zeros((n, k, pitch), dtype=_dtype(case["dtype"]), device=DEV)[:, :, :v]
    draft.copy_(q)
    noise = torch.rand((n, k, v), generator=g, device=DEV).clamp_(min=1e-30).log_().neg_().clamp_(min=1e-30).log_().neg_()
    tokens = (draft.float() / case["temperature"] + noise).argmax(-1) if k else torch.zeros((n, 0), dtype=torch.int64, device=DEV)
    lengths = torch.randint(0, k + 1, (n,), generator=g, device=DEV)
    lengths = torch.where(torch.rand((n,), generator=g, device=DEV) < 0.75, torch.full_like(lengths, k), lengths).to(torch.int32)
    return dict(target=target, draft=draft if case["draft"] == "logits" else None, tokens=tokens, lengths=lengths,
                accept_u=torch.rand((n, k), generator=g, device=DEV),
                sample_u=torch.rand((n,), generator=g, device=DEV, dtype=torch.float64))


def _prepare_norm(case, g):
    n, d, dt = case["rows"], case["d_model"], case["dtype"]
    s = dict(residual=_rows(g, n, d, case["residual"], 4.0), block=_rows(g, n, d, dt, 1.5),
             post=_rows(g, 1, d, dt, 0.1, 1.0)[0] if case["post"] else None, pre=_rows(g, 1, d, dt, 0.1, 1.0)[0], gate=None)
    if case["gate"] != "none":
        s["gate"] = _rows(g, n if case["gate"] == "full" else 1, d, dt, 1.0).sigmoid_()
        if case["gate"] == "row":
            s["gate"] = s["gate"][0]
    if case["path"] == "norm_bwd":
        s["grad_hidden"] = _rows(g, n, d, dt, 0.01)
        s["grad_residual_out"] = _rows(g, n, d, case["residual"], 0.01)
    return s


def _sizes(case):
    d = case["d_model"]
    sizes = [case["vocab"] * d] if case["vocab"] else []
    for _ in range(case["layers"]):  # two norms, the attention's four matrices, the feed-forward block's two
        sizes += [d, d * d, d * d, d * d, d * d, d, 4 * d * d, 4 * d * d]
    return sizes + [d]


def _matrix(case):
    """Which of the tensors are matrices: those alone decay."""
    return [n != case["d_model"] for n in _sizes(case)]


def _starts(case):
    """Where the tensors begin in the buffer that holds them all, and its length."""
    at, starts = 0, []
    for n in _sizes(case):
        starts.append(at)
        at += (n + case["pad"] - 1) // case["pad"] * case["pad"]
    return starts, at


def _prepare_tensors(case, g):
    starts, total = _starts(case)
    sizes = _sizes(case)

    def flat(scale, dtype=torch.float32):
        t = torch.empty(total, dtype=torch.float32, device=DEV).normal_(generator=g).mul_(scale)
        for a, n, b in zip(starts, sizes, starts[1:] + [total]):
            t[a + n:b] = 0.0  # between tensors
        return t if dtype == torch.float32 else t.to(dtype)

    s = dict(grad=flat(2e-5, _dtype(case["grad"])))
    for a, n, k in zip(starts, sizes, range(len(sizes))):  # layers differ
        s["grad"][a:a + n].mul_(2.0 ** (k % 5 - 2))
    if case["path"] == "clip":
        return s
    s["clip"] = torch.tensor([0.25, 0.4], device=DEV)  # norm and coefficient
    master = flat(0.02)
    s["master"] = master if case["param"] == "master" else None
    s["param"] = master if case["param"] == "f32" else master.to(torch.bfloat16)
    m, r = flat(1e-5), flat(2e-5).abs_()
    if case["bits"] == 8:
        s["m"], s["m_scale"] = _quantise(m)
        s["r"], s["r_scale"] = _quantise(r, keep=True)
    else:
        s["m"], s["v"] = m, r.square_()
    return s


def prepare(case, seed):
    g = _gen(seed)
    if case["path"] == "verify":
        return dict(case=case, **_prepare_verify(case, g))
    if case["path"].startswith("norm"):
        return dict(case=case, **_prepare_norm(case, g))
    s = dict(case=case, **_prepare_tensors(case, g))
    if own:  # which tensors there are: a trainer says so once
        s["plan"] = _plan(s, case)
    return s


def _plan(s, case):
    import paper_2505_07291_amd as grpo

    def cut(t, per=1):
        return None if t is None else [t[a // per:(a + n + per - 1) // per] for a, n in zip(*(_starts(case)[0], _sizes(case)))]

    if case["path"] == "clip":
        return grpo.grpo_optim_plan(None, cut(s["grad"]))
    eight = case["bits"] == 8
    return grpo.grpo_optim_plan(cut(s["param"]), cut(s["grad"]), cut(s["m"]), cut(s["r"] if eight else s["v"]), masters=cut(s["master"]),
                                exp_avg_scales=cut(s["m_scale"], QUANT) if eight else None,
                                exp_avg_sq_scales=cut(s["r_scale"], QUANT) if eight else None,
                                weight_decay=[DECAY if m else 0.0 for m in _matrix(case)])


# ---- plain forms ---------------------------------------------------------------------------------------------------

def _log_softmax(z):
    z = z - z.amax(-1, keepdim=True)
    return z - z.exp().sum(-1, keepdim=True).log()


def _plain_verify(s, case):
    n, k, v = case["batch"], case["drafts"], case["vocab"]
    # in 64 bits: a token next to a border of the cumulative sums, or a ratio next to its random number
    lp = _log_softmax(s["target"].double() / case["temperature"])
    place = torch.arange(k + 1, device=DEV)
    if k:
        y = s["tokens"][:, :, None]
        p = lp[:, :k].gather(2, y)[:, :, 0].exp()
        if s["draft"] is not None:
            q = _log_softmax(s["draft"].double() / case["temperature"]).exp()
            qy = q.gather(2, y)[:, :, 0]
        else:
            q = torch.zeros((n, k, v), dtype=torch.float64, device=DEV).scatter_(2, y, 1.0)
            qy = 1.0
        taken = (s["accept_u"].double() * qy < p) & (place[:k] < s["lengths"][:, None])
        accepted = taken.to(torch.int64).cumprod(1).sum(1)
    else:
        accepted = torch.zeros(n, dtype=torch.int64, device=DEV)
    row = accepted[:, None, None].expand(n, 1, v)
    p = lp.gather(1, row)[:, 0].exp()
    w = p
    if k:
        rest = (p - q.gather(1, row.clamp(max=k - 1))[:, 0]).clamp(min=0.0)
        refused = (accepted < s["lengths"])[:, None] & (rest.sum(1, keepdim=True) > 0)
        w = torch.where(refused, rest, p)
    c = w.cumsum(1)
    token = (c <= s["sample_u"][:, None] * c[:, -1:]).sum(1).clamp(max=v - 1)
    out = torch.where(place < accepted[:, None], torch.cat([s["tokens"], token[:, None]], 1), token[:, None])
    logprobs = lp.gather(2, out[:, :, None])[:, :, 0]
    emitted = place <= accepted[:, None]
    return torch.where(emitted, out, -1), accepted.to(torch.int32), torch.where(emitted, logprobs, 0.0).float()


def _rms(x):
    return (x.square().mean(-1, keepdim=True) + EPS).rsqrt()


def _plain_norm_fwd(s, case):
    x, branch = s["residual"].float(), s["block"].float()
    if s["post"] is not None:
        branch = branch * _rms(branch) * s["post"].float()
    if s["gate"] is not None:
        branch = branch * s["gate"].float()
    x = x + RESIDUAL_SCALE * branch
    return x.to(s["residual"].dtype), (x * _rms(x) * s["pre"].float()).to(s["block"].dtype)


def _plain_norm_bwd(s, case):
    dt, x, f = s["block"].dtype, s["residual"].float(), s["block"].float()
    dh = s["grad_hidden"].float()
    r = _rms(x)
    y = x * r
    a = dh * s["pre"].float()
    dx = s["grad_residual_out"].float() + r * (a - y * (a * y).mean(-1, keepdim=True))
    grad_pre = (dh * y).sum(0)
    r = _rms(f) if s["post"] is not None else 1.0
    y = f * r
    t = RESIDUAL_SCALE * dx
    grad_gate = grad_post = None
    w = s["post"].float() if s["post"] is not None else 1.0
    if s["gate"] is not None:
        grad_gate = t * (y * w)
        grad_gate = grad_gate.sum(0) if s["gate"].dim() == 1 else grad_gate.to(dt)
        t = t * s["gate"].float()
    if s["post"] is not None:
        grad_post = (t * y).sum(0)
        t = t * w
        t = r * (t - y * (t * y).mean(-1, keepdim=True))
    return dx.to(s["residual"].dtype), t.to(dt), grad_gate, grad_post, grad_pre


def _plain_clip(s, case):
    norm = s["grad"].double().square().sum().sqrt()
    return torch.stack([norm, torch.where(norm <= MAX_NORM, 1.0, MAX_NORM / norm)]).float()


def _quantise(x, keep=False):
    """Values in 8 bits (e4m3) and a power of two for each QUANT of them; keep: positive ones stay positive."""
    x = x.view(-1, QUANT)
    bits = torch.where(x.isfinite(), x, 0.0).abs().amax(1).view(torch.int32)
    # the least power of two under which the largest value is at most 448 = 1.75 * 2^8
    e = (bits >> 23) - 127 - 8 + ((bits & 0x7fffff) > 0x600000).to(torch.int32)
    e = e.clamp(min=-126)
    y = x * ((127 - e) << 23).view(torch.float32)[:, None]
    if keep:
        y = torch.where((x > 0) & (y < TINY_CODE), TINY_CODE, y)
    return y.to(torch.float8_e4m3fn).view(-1), ((e + 127) << 23).view(torch.float32)


def _plain_adamw(s, case):
    starts, total = _starts(case)
    decay = torch.tensor([1.0 - LR * DECAY if m else 1.0 for m in _matrix(case)], dtype=torch.float32, device=DEV).split(1)
    decay = torch.cat([d.expand(b - a) for d, a, b in zip(decay, starts, starts[1:] + [total])])
    g = s["grad"].float() * s["clip"][1]
    eight = case["bits"] == 8
    if eight:
        m = (s["m"].float().view(-1, QUANT) * s["m_scale"][:, None]).view(-1)
        v = (s["r"].float().view(-1, QUANT) * s["r_scale"][:, None]).view(-1).square()
    else:
        m, v = s["m"], s["v"]
    # every product and sum rounded by itself: the moments in 8 bits are rounded from the same 32 on either side
    m = m * BETA1 + g * (1.0 - BETA1)
    v = v * BETA2 + g * g * (1.0 - BETA2)
    r = v.sqrt()
    step = m / (r * (1.0 / math.sqrt(1.0 - BETA2 ** STEP)) + ADAM_EPS)
    p = (s["master"] if s["master"] is not None else s["param"]).float() * decay - step * (LR / (1.0 - BETA1 ** STEP))
    s["param"].copy_(p)
    if s["master"] is not None:
        s["master"].copy_(p)
    if eight:
        for name, (codes, scale) in (("m", _quantise(m)), ("r", _quantise(r, keep=True))):
            s[name].copy_(codes)
            s[name + "_scale"].copy_(scale)
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    return _state(s)


def _state(s):
    return {k: s[k] for k in ("param", "master", "m", "v", "r", "m_scale", "r_scale") if s.get(k) is not None}


_PLAIN = dict(verify=_plain_verify, norm_fwd=_plain_norm_fwd, norm_bwd=_plain_norm_bwd, clip=_plain_clip, adamw=_plain_adamw)


def run(s):
    case = s["case"]
    path = case["path"]
    if not own:
        return _PLAIN[path](s, case)
    import paper_2505_07291_amd as grpo
    if path == "verify":
        return grpo.grpo_verify_drafts(s["target"], s["draft"], s["tokens"], s["accept_u"], s["sample_u"], s["lengths"],
                                       temperature=case["temperature"], draft_temperature=case["temperature"])
    if path == "norm_fwd":
        return grpo.grpo_block_norm_fwd(s["residual"], s["block"], s["post"], s["gate"], s["pre"], residual_scale=RESIDUAL_SCALE, eps=EPS)
    if path == "norm_bwd":
        return grpo.grpo_block_norm_bwd(s["residual"], s["block"], s["post"], s["gate"], s["pre"], s["grad_hidden"],
                                        s["grad_residual_out"], residual_scale=RESIDUAL_SCALE, eps=EPS)
    if path == "clip":
        return grpo.grpo_grad_norm(s["plan"], max_norm=MAX_NORM)
    grpo.grpo_adamw_step(s["plan"], STEP, LR, BETA1, BETA2, ADAM_EPS, clip=s["clip"])
    return _state(s)


# ---- what a pass cannot do without -----------------------------------------------------------------------------------

def work(case):
    path = case["path"]
    if path == "verify":
        n, k, v, size = case["batch"], case["drafts"], case["vocab"], _bytes(case["dtype"])
        # the rows up to the first draft that is not accepted: about four in five are, an n-gram's guess hardly ever
        a = 0.8 if case["draft"] == "logits" else 0.05
        rows = sum(a ** i for i in range(k + 1))
        rows += sum(a ** i for i in range(k)) if case["draft"] == "logits" else 0
        return dict(bytes=n * (rows * v * size + (k + 1) * 24 + 12), flops=4.0 * n * rows * v)
    if path.startswith("norm"):
        n, d, size, res = case["rows"], case["d_model"], _bytes(case["dtype"]), _bytes(case["residual"])
        gate = 1 if case["gate"] == "full" else 0
        if path == "norm_fwd":
            return dict(bytes=n * d * (2 * res + (2 + gate) * size), flops=10.0 * n * d)
        return dict(bytes=n * d * (3 * res + (3 + 2 * gate) * size), flops=30.0 * n * d)
    values = sum(_sizes(case))
    if path == "clip":
        return dict(bytes=values * _bytes(case["grad"]), flops=2.0 * values)
    per = _bytes(case["grad"]) + dict(f32=8, bf16=4, master=10)[case["param"]] + (4 if case["bits"] == 8 else 16)
    return dict(bytes=values * per, flops=15.0 * values)


# ---- the definitions, in 64 bits -------------------------------------------------------------------------------------

def _exact_verify(s, case):
    import numpy as np
    n, k, v, temp = case["batch"], case["drafts"], case["vocab"], case["temperature"]
    target = s["target"].float().cpu().numpy()
    draft = None if s["draft"] is None else s["draft"].float().cpu().numpy()
    drafted, lengths = s["tokens"].cpu().numpy(), s["lengths"].cpu().numpy()
    u, su = s["accept_u"].double().cpu().numpy(), s["sample_u"].cpu().numpy()

    def normed(row):
        z = row.astype(np.float64) / temp
        e = np.exp(z - z.max())
        return e / e.sum()

    tokens, logprobs = np.full((n, k + 1), -1, np.int64), np.zeros((n, k + 1))
    accepted = np.zeros(n, np.int32)
    for b in range(n):
        for i in range(k + 1):
            p = normed(target[b, i])
            w = p
            if i < lengths[b]:
                y = drafted[b, i]
                q = np.eye(1, v, y)[0] if draft is None else normed(draft[b, i])
                if u[b, i] * q[y] < p[y]:
                    tokens[b, i], logprobs[b, i] = y, np.log(p[y])
                    continue
                w = np.maximum(p - q, 0.0)
                w = w if w.any() else p
            c = np.cumsum(w)
            y = min(int(np.searchsorted(c, su[b] * c[-1], side="right")), v - 1)
            tokens[b, i], logprobs[b, i], accepted[b] = y, np.log(p[y]), i
            break
    return tokens, accepted, logprobs


def _exact_forward(x, f, post, gate, pre):
    def rms_norm(t):
        return t / torch.sqrt(torch.mean(t ** 2, dim=1, keepdim=True) + EPS)

    branch = f if post is None else rms_norm(f) * post
    out = x + RESIDUAL_SCALE * (branch if gate is None else gate * branch)
    return out, rms_norm(out) * pre


def _exact_norm(s, case):
    wide = lambda t: None if t is None else t.double()  # noqa: E731
    if case["path"] == "norm_fwd":
        return _exact_forward(*(wide(s[k]) for k in ("residual", "block", "post", "gate", "pre")))
    # automatic differentiation; the sum is given, so what is added to the branch is what leaves it there
    leaves = {k: s[k].double().requires_grad_() for k in ("block", "post", "gate", "pre") if s[k] is not None}
    with torch.no_grad():
        x = s["residual"].double()
        x = x - (_exact_forward(x, *(wide(s[k]) for k in ("block", "post", "gate", "pre")))[0] - x)
    x.requires_grad_()
    out, hidden = _exact_forward(x, *(leaves.get(k) for k in ("block", "post", "gate", "pre")))
    names = [k for k in ("block", "gate", "post", "pre") if k in leaves]
    got = torch.autograd.grad([out, hidden], [x] + [leaves[k] for k in names], [s["grad_residual_out"].double(), s["grad_hidden"].double()])
    got = dict(zip(["x"] + names, got))
    return [got.get(k) for k in ("x", "block", "gate", "post", "pre")]


def _exact_clip(s, case):
    total = math.fsum(float(torch.linalg.vector_norm(part.double())) ** 2 for part in s["grad"].split(1 << 24))
    norm = math.sqrt(total)
    return torch.tensor([norm, min(1.0, MAX_NORM / norm)], dtype=torch.float64)


def _exact_adamw(s, case):
    out = {}
    g = s["grad"].double() * float(s["clip"][1])
    eight = case["bits"] == 8
    per = lambda t: t.double().repeat_interleave(QUANT)  # noqa: E731
    m = s["m"].float().double() * per(s["m_scale"]) if eight else s["m"].double()
    m = torch.lerp(g, m, BETA1)
    v = (s["r"].float().double() * per(s["r_scale"])) ** 2 if eight else s["v"].double()
    v = torch.lerp(g ** 2, v, BETA2)
    p = (s["param"] if s["master"] is None else s["master"]).double()
    for a, n, matrix in zip(_starts(case)[0], _sizes(case), _matrix(case)):
        part = slice(a, a + n)
        if matrix:
            p[part] -= LR * DECAY * p[part]
        p[part] -= LR * (m[part] / (1 - BETA1 ** STEP)) / (torch.sqrt(v[part] / (1 - BETA2 ** STEP)) + ADAM_EPS)
    out["param"] = p
    if s["master"] is not None:
        out["master"] = p
    if not eight:
        return dict(out, m=m, v=v)
    for name, t in (("m", m), ("r", v.sqrt())):  # what the codes stand for, before they are rounded to it
        top = t.view(-1, QUANT).abs().amax(1)
        # where the largest value is a border's within 32 bits (products of 8-bit values and bf16 gradients often are), either scale is right
        scale = torch.exp2(torch.ceil(torch.log2(top / 448.0) - 3e-7).clamp(min=-126))
        out[name], out[name + "_scale"] = t / scale.repeat_interleave(QUANT), None
    return out


def exact(case, seed):
    s = prepare(case, seed)
    path = case["path"]
    if path == "verify":
        return _exact_verify(s, case)
    return dict(norm_fwd=_exact_norm, norm_bwd=_exact_norm, clip=_exact_clip, adamw=_exact_adamw)[path](s, case)
