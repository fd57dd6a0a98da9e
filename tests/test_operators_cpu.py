"""Verification of drafted tokens, a block's norms, the gradients' norm and AdamW without a GPU: every bad argument gets its
status code before the device is touched, and the table of an optimiser's tensors, which is made on the host, is what was asked for."""
import ctypes

import pytest
import torch

import paper_2505_07291_amd as grpo
from paper_2505_07291_amd.binding import _OptimPlan, _OptimTensor

OK, NULL, SHAPE, DTYPE, ALIGN, PARAM, WORKSPACE, HIP, CAPACITY, OVERLAP = range(10)
P = 0x7F0000001000  # a fake, 256-byte aligned, non-null "device pointer": validation never dereferences
NAN, INF = float("nan"), float("inf")


def test_the_new_status_has_a_text():
    assert grpo.status_string(OVERLAP) not in ("unknown status", grpo.status_string(CAPACITY))
    assert grpo.status_string(10) == "unknown status"


VERIFY = dict(target=P, tb=4096, ts=1024, draft=P, db=4096, ds=1024, dtype=1, n=4, k=3, V=1000, tokens=P, u=P, v=P, lengths=P, t=1.0, td=1.0,
              out=P, acc=P, lp=P, ws=P, bytes=1 << 24, stream=None)


@pytest.mark.parametrize("over,expect", [
    (dict(dtype=2), DTYPE), (dict(dtype=-1), DTYPE),
    (dict(n=-1), SHAPE), (dict(n=1 << 31), SHAPE), (dict(n=1 << 24, k=0), SHAPE), (dict(n=1 << 19, k=64), SHAPE), (dict(k=-1), SHAPE), (dict(k=65), SHAPE), (dict(V=0), SHAPE),
    (dict(V=(1 << 28) + 1), SHAPE), (dict(ts=992), SHAPE), (dict(ds=992), SHAPE), (dict(tb=-8), SHAPE), (dict(db=-8), SHAPE),
    (dict(t=0.0), PARAM), (dict(t=-1.0), PARAM), (dict(t=NAN), PARAM), (dict(t=INF), PARAM), (dict(t=1e-31), PARAM), (dict(td=1e31), PARAM), (dict(td=0.0), PARAM), (dict(td=NAN), PARAM),
    (dict(target=None), NULL), (dict(tokens=None), NULL), (dict(u=None), NULL), (dict(v=None), NULL), (dict(out=None), NULL),
    (dict(acc=None), NULL), (dict(lp=None), NULL),
    (dict(target=P + 8), ALIGN), (dict(ts=1001), ALIGN), (dict(tb=4097), ALIGN), (dict(draft=P + 4), ALIGN), (dict(ds=1004), ALIGN),
    (dict(db=4100), ALIGN), (dict(dtype=0, ts=1002), ALIGN),
    (dict(ws=None), WORKSPACE), (dict(ws=P + 16), WORKSPACE), (dict(bytes=100), WORKSPACE),
    (dict(n=0, target=None, tokens=None, ws=None), OK),
])
def test_verify_refusals(over, expect):
    a = dict(VERIFY, **over)
    assert grpo.lib().grpo_verify_drafts(*a.values()) == expect


def test_verify_workspace():
    f = grpo.lib().grpo_verify_workspace_bytes
    assert [f(-1, 3, 1000, 1), f(4, -1, 1000, 1), f(4, 65, 1000, 1), f(4, 3, 0, 1), f(4, 3, (1 << 28) + 1, 1), f(4, 3, 1000, 5),
            f(1 << 30, 64, 1 << 28, 1)] == [0] * 7
    for n, k, v in ((0, 0, 1), (1, 0, 1), (1, 64, 1 << 28), ((1 << 24) - 1, 0, 100), (96, 5, 152064), (1000, 8, 300007), (1 << 20, 0, 1000)):
        for dtype in (0, 1):
            need = f(n, k, v, dtype)
            # sums to each part of a row, at most 1024 parts
            assert 0 < need <= 1024 + n * (k + 2) * 4 + n * 1024 * (2 * k * 8 + 44)
            a = dict(VERIFY, n=n, k=k, V=v, dtype=dtype, ts=(v + 7) // 8 * 8, ds=(v + 7) // 8 * 8, bytes=need - 1)
            if n:
                assert grpo.lib().grpo_verify_drafts(*a.values()) == WORKSPACE


FWD = dict(x=P, xs=520, rt=0, f=P, fs=520, w1=P, g=P, gs=520, w2=P, dt=1, n=4, d=513, scale=1.0, eps=1e-6, xo=P, xos=520, h=P, hs=520, stream=None)
BWD = dict(x=P, xs=520, rt=0, f=P, fs=520, w1=P, g=P, gs=520, w2=P, dt=1, n=4, d=513, scale=1.0, eps=1e-6, dh=P, dhs=520, dxo=P, dxos=520,
           dx=P, dxs=520, df=P, dfs=520, dg=P, dgs=520, dw1=P, dw2=P, acc=0, ws=P, bytes=1 << 20, stream=None)
BOTH = [
    (dict(rt=2), DTYPE), (dict(dt=3), DTYPE), (dict(rt=1, dt=0), DTYPE),
    (dict(n=-1), SHAPE), (dict(d=0), SHAPE), (dict(d=(1 << 20) + 1), SHAPE), (dict(xs=512), SHAPE), (dict(fs=512), SHAPE), (dict(gs=512), SHAPE),
    (dict(gs=-8), SHAPE),
    (dict(scale=NAN), PARAM), (dict(scale=INF), PARAM), (dict(eps=-1e-9), PARAM), (dict(eps=NAN), PARAM), (dict(eps=INF), PARAM),
    (dict(f=None), NULL), (dict(f=None, w1=None), NULL), (dict(f=None, g=None), NULL), (dict(x=None), NULL),
    (dict(x=P + 4), ALIGN), (dict(f=P + 8), ALIGN), (dict(w1=P + 2), ALIGN), (dict(w2=P + 2), ALIGN), (dict(g=P + 8), ALIGN),
    (dict(xs=517), ALIGN), (dict(fs=516), ALIGN), (dict(gs=516), ALIGN), (dict(rt=1, xs=516), ALIGN),
]


@pytest.mark.parametrize("over,expect", BOTH + [
    (dict(xo=None), NULL), (dict(h=None), NULL), (dict(w2=None), NULL), (dict(f=None, w1=None, g=None, gs=0), NULL),
    (dict(f=None, w1=None, g=None, gs=0, w2=None, xo=None, h=None), NULL),
    (dict(xos=512), SHAPE), (dict(hs=512), SHAPE), (dict(xo=P + 4), ALIGN), (dict(h=P + 4), ALIGN), (dict(hs=516), ALIGN), (dict(n=0), OK),
])
def test_block_norm_forward_refusals(over, expect):
    assert grpo.lib().grpo_block_norm_fwd(*dict(FWD, **over).values()) == expect


@pytest.mark.parametrize("over,expect", BOTH + [
    (dict(dh=None), NULL), (dict(dx=None), NULL), (dict(df=None), NULL), (dict(dg=None), NULL), (dict(dw1=None), NULL), (dict(dw2=None), NULL),
    (dict(w1=None), NULL), (dict(w2=None), NULL), (dict(g=None), NULL), (dict(gs=0, dg=None), NULL),
    (dict(w2=None, dw2=None, dh=None, x=None, dxo=None), NULL),  # nothing that a gradient could come from
    (dict(dhs=512), SHAPE), (dict(dxos=512), SHAPE), (dict(dxs=512), SHAPE), (dict(dfs=512), SHAPE), (dict(dgs=512), SHAPE),
    (dict(dh=P + 4), ALIGN), (dict(dxo=P + 4), ALIGN), (dict(dx=P + 4), ALIGN), (dict(df=P + 4), ALIGN), (dict(dg=P + 4), ALIGN),
    (dict(dgs=516), ALIGN),
    (dict(ws=None), WORKSPACE), (dict(ws=P + 128), WORKSPACE), (dict(bytes=4096), WORKSPACE),
])
def test_block_norm_backward_refusals(over, expect):
    assert grpo.lib().grpo_block_norm_bwd(*dict(BWD, **over).values()) == expect


def test_block_norm_workspace():
    f = grpo.lib().grpo_block_norm_workspace_bytes
    assert f(-1, 8) == f(8, 0) == f(8, -1) == f(8, (1 << 20) + 1) == 0
    assert 0 < f(0, 5120) <= 4096
    for n, d in ((1, 1), (100, 5120), (1 << 40, 1 << 20)):
        assert f(n, d) % 256 == 0 and 0 < f(n, d) <= 512 + 1024 * 2 * 4 * (d + 64)


def tensor(base=P, n=1000, param=0, grad=0, bits=32, master=False, **over):
    """A tensor whose arrays lie 64 KB apart from `base` on."""
    at = [base + 65536 * i for i in range(7)]
    t = dict(param=at[0], master=at[1] if master else None, grad=at[2], exp_avg=at[3], exp_avg_sq=at[4], exp_avg_scale=at[5] if bits == 8 else None,
             exp_avg_sq_scale=at[6] if bits == 8 else None, n=n, weight_decay=0.1, param_dtype=param, grad_dtype=grad, state_bits=bits, reserved=0)
    t.update(over)
    return _OptimTensor(*t.values())


def build(tensors, spare=0, table=True, out=True):
    L = grpo.lib()
    array = (_OptimTensor * max(1, len(tensors)))(*tensors)
    need = L.grpo_optim_plan_bytes(array, len(tensors))
    buffer = ctypes.create_string_buffer(max(1, need))
    plan = _OptimPlan()
    rc = L.grpo_optim_plan_build(array, len(tensors), ctypes.addressof(buffer) if table else None, max(0, need + spare), ctypes.byref(plan) if out else None)
    return rc, plan, need


@pytest.mark.parametrize("over,expect", [
    (dict(), OK), (dict(bits=8), OK), (dict(param=1), OK), (dict(param=1, master=True), OK), (dict(grad=1), OK),
    (dict(param=2), DTYPE), (dict(param=-1), DTYPE), (dict(grad=5), DTYPE), (dict(bits=16), DTYPE), (dict(master=True), DTYPE),
    (dict(n=-1), SHAPE), (dict(n=(1 << 40) + 1), SHAPE), (dict(n=1 << 36), SHAPE), (dict(weight_decay=NAN), PARAM), (dict(weight_decay=INF), PARAM),
    (dict(exp_avg=None), NULL), (dict(exp_avg_sq=None), NULL), (dict(bits=8, exp_avg_scale=None), NULL),
    (dict(bits=8, exp_avg_sq_scale=None), NULL), (dict(exp_avg_scale=P), NULL),
    (dict(grad=0, exp_avg=P + 1), ALIGN), (dict(exp_avg_sq=P + 65536 * 4 + 2), ALIGN), (dict(bits=8, exp_avg_scale=P + 65536 * 5 + 2), ALIGN),
    (dict(exp_avg=P), OVERLAP), (dict(exp_avg_sq=P + 3996), OVERLAP), (dict(exp_avg_sq=P + 4000), OK),
    (dict(bits=8, exp_avg_scale=P + 65536 * 4 + 996), OVERLAP), (dict(n=20000), OVERLAP),
])
def test_plan_refusals(over, expect):
    assert build([tensor(P + (1 << 24)), tensor(**over)])[0] == expect


def test_plan_of_addresses():
    """The arrays themselves: a parameter at an odd address, a gradient that two tensors share, one that is a parameter too."""
    def at(**over):
        t = tensor()
        for k, v in over.items():
            setattr(t, k, v)
        return t

    assert build([at(param=P + 2)])[0] == ALIGN
    assert build([at(grad=P + 65536 * 2 + 1)])[0] == ALIGN
    assert build([at(grad=None)])[0] == NULL
    assert build([at(param=None)])[0] == NULL  # moments without a parameter
    assert build([at(param=P + 4)])[0] == OK
    a, b = tensor(), tensor(P + (1 << 24))
    b.grad = a.grad
    assert build([a, b])[0] == OK
    b.grad = a.param
    assert build([a, b])[0] == OVERLAP
    assert build([a, a])[0] == OVERLAP


def test_plan_sizes_and_refused_buffers():
    sizes = [1, 8192, 8193, 0, 16384]
    tensors = [tensor(P + (i << 24), n) for i, n in enumerate(sizes)]
    rc, plan, need = build(tensors)
    assert rc == OK and plan.n_tensors == 5 and plan.n_chunks == sum(-(-n // 4096) for n in sizes) and plan.has_params == 1
    assert need % 256 == 0 and need >= 5 * 88 + 8 * plan.n_chunks
    assert build(tensors, spare=-1)[0] == WORKSPACE
    assert build(tensors, table=False)[0] == NULL and build(tensors, out=False)[0] == NULL
    rc, plan, _ = build([])
    assert rc == OK and (plan.n_tensors, plan.n_chunks) == (0, 0)
    only = tensor()
    for name in ("param", "exp_avg", "exp_avg_sq"):
        setattr(only, name, None)
    rc, plan, _ = build([only])
    assert rc == OK and plan.has_params == 0
    L = grpo.lib()
    assert L.grpo_optim_plan_bytes(None, 3) == 0 and L.grpo_optim_plan_bytes(None, -1) == 0
    assert L.grpo_optim_plan_build(None, -1, ctypes.addressof(plan), 1 << 20, ctypes.byref(plan)) == SHAPE


@pytest.mark.parametrize("over,expect", [
    (dict(plan=None), NULL), (dict(table=None), NULL), (dict(table=P + 64), ALIGN), (dict(max_norm=NAN), PARAM), (dict(out=None), NULL),
    (dict(ws=None), WORKSPACE), (dict(ws=P + 8), WORKSPACE), (dict(bytes=100), WORKSPACE), (dict(chunks=-1), SHAPE), (dict(tensors=-1), SHAPE),
])
def test_grad_norm_refusals(over, expect):
    a = dict(plan=1, table=P, max_norm=0.1, out=P, ws=P, bytes=1 << 20, stream=None, tensors=3, chunks=7)
    a.update(over)
    plan = _OptimPlan(a["tensors"], a["chunks"], 1, 0)
    args = [ctypes.byref(plan) if a["plan"] else None] + [a[k] for k in ("table", "max_norm", "out", "ws", "bytes", "stream")]
    assert grpo.lib().grpo_grad_norm(*args) == expect


@pytest.mark.parametrize("over,expect", [
    (dict(plan=None), NULL), (dict(table=None), NULL), (dict(table=P + 64), ALIGN), (dict(params=0), NULL), (dict(step=0), PARAM), (dict(step=-3), PARAM),
    (dict(lr=NAN), PARAM), (dict(lr=INF), PARAM), (dict(b1=1.0), PARAM), (dict(b1=-0.1), PARAM), (dict(b1=NAN), PARAM), (dict(b2=1.0), PARAM),
    (dict(b2=-0.1), PARAM), (dict(eps=-1.0), PARAM), (dict(eps=NAN), PARAM), (dict(eps=INF), PARAM),
    (dict(chunks=0, tensors=0, params=0, table=None), OK),
])
def test_adamw_refusals(over, expect):
    a = dict(plan=1, table=P, step=1, step_at=None, lr=0.1, lr_at=None, b1=0.9, b2=0.999, eps=1e-8, clip=None, stream=None, tensors=3, chunks=7, params=1)
    a.update(over)
    plan = _OptimPlan(a["tensors"], a["chunks"], a["params"], 0)
    args = [ctypes.byref(plan) if a["plan"] else None] + [a[k] for k in ("table", "step", "step_at", "lr", "lr_at", "b1", "b2", "eps", "clip", "stream")]
    assert grpo.lib().grpo_adamw_step(*args) == expect


def test_host_tensors_are_refused():
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError, match="device tensor"):
        grpo.grpo_block_norm_fwd(x, pre_weight=x[0])
    with pytest.raises(ValueError, match="device tensor"):
        grpo.grpo_block_norm_bwd(x, pre_weight=x[0], grad_hidden=x)
    with pytest.raises(ValueError, match="device tensor"):
        grpo.grpo_verify_drafts(x[None], None, None, None, torch.zeros(1, dtype=torch.float64))
    with pytest.raises(ValueError, match="device tensor"):
        grpo.grpo_optim_plan([x], [x.clone()], [x.clone()], [x.clone()])
    with pytest.raises(ValueError, match="no tensors"):
        grpo.grpo_optim_plan([], [], [], [])
