"""Refusals of the norm, loss and optimizer calls: the C entry points return before any device work, the Python calls raise."""
import ctypes

import pytest
import torch

import paper_2104_06700_amd as gnn

BAD, OK = gnn.GNN_ERR_INVALID_ARG, gnn.GNN_OK
P = ctypes.c_void_p(256)  # never dereferenced: every call below returns before touching memory
Q = ctypes.c_void_p(512)


def test_struct_layouts_match_the_header():
    # gnn_norm_opts: 3 x int32, float, 4 x int64, 2 pointers, int64; gnn_loss_opts: 3 x int32, float, 2 x int64, 2 pointers, int64
    assert ctypes.sizeof(gnn.GnnNormOpts) == 16 + 32 + 16 + 8
    assert ctypes.sizeof(gnn.GnnLossOpts) == 16 + 16 + 16 + 8
    # gnn_adamw_tensor: 7 pointers, int64, 2 x int32, float, int32; gnn_adamw_opts: 4 doubles, 2 x int64, 2 pointers
    assert ctypes.sizeof(gnn.GnnAdamWTensor) == 56 + 8 + 16
    assert ctypes.sizeof(gnn.GnnAdamWOpts) == 32 + 16 + 16


def _norm(backward=False, x=P, y=Q, n=100, c=64, g=8, b=1, ptr=None, stats=P, workspace=1 << 30, opts=True, **kw):
    o = gnn.GnnNormOpts(eps=1e-5, workspace=256, workspace_bytes=workspace)
    for k, v in kw.items():
        setattr(o, k, v)
    lib = gnn.load_library()
    o = ctypes.byref(o) if opts else None
    if backward:
        return lib.gnn_group_norm_bwd(x, None, None, stats, stats, P, ptr, y, None, None, n, c, g, b, o)
    return lib.gnn_group_norm_fwd(x, None, None, ptr, y, stats, stats, n, c, g, b, o)


@pytest.mark.parametrize("kw", [
    dict(n=-1), dict(c=-64), dict(g=0), dict(g=-8), dict(g=7), dict(b=0), dict(b=-1), dict(b=3), dict(n=1 << 31), dict(c=(1 << 24) + 8),
    dict(dtype=2), dict(dtype=-1), dict(act=3), dict(act=-1), dict(eps=-1.0), dict(eps=float("nan")), dict(ldx=63), dict(ldy=63), dict(lddx=63),
    dict(ldx=-64), dict(max_sample_rows=-1), dict(x=None), dict(y=P), dict(stats=None), dict(workspace=16), dict(workspace=0), dict(opts=False)])
def test_norm_refuses(kw):
    assert _norm(**kw) == BAD
    if "y" not in kw:  # (the backward call's dX may be missing, and dY is at P)
        assert _norm(backward=True, **kw) == BAD
    else:
        assert _norm(backward=True, y=P) == BAD


def test_norm_workspace_must_be_aligned_and_empty_calls_succeed():
    o = gnn.GnnNormOpts(workspace=264, workspace_bytes=1 << 30)
    assert gnn.load_library().gnn_group_norm_fwd(P, None, None, None, Q, P, P, 100, 64, 8, 1, ctypes.byref(o)) == BAD
    assert _norm(n=0) == OK and _norm(c=0, g=1) == OK and _norm(n=0, b=0, x=None, y=None, stats=None, workspace=0) == OK
    assert _norm(backward=True, c=0, g=1) == OK
    assert _norm(backward=True, y=None) == OK  # no gradient asked for
    assert gnn.gnn_group_norm_workspace_bytes(0, 64, 8) == 0 and gnn.gnn_group_norm_workspace_bytes(-5, 64, 8) == 0
    assert gnn.gnn_group_norm_workspace_bytes(100, 64, 8, 4, True) >= gnn.gnn_group_norm_workspace_bytes(100, 64, 8, 4) > 0


def _loss(x=P, labels=P, loss=P, dx=Q, n=10, c=5, workspace=1 << 20, opts=True, **kw):
    o = gnn.GnnLossOpts(scale=1.0, workspace=256, workspace_bytes=workspace)
    for k, v in kw.items():
        setattr(o, k, v)
    return gnn.load_library().gnn_softmax_xent(x, labels, loss, dx, None, n, c, ctypes.byref(o) if opts else None)


@pytest.mark.parametrize("kw", [
    dict(n=-1), dict(c=-1), dict(n=1 << 31), dict(c=1 << 31), dict(dtype=2), dict(reduction=2), dict(reduction=-1), dict(ldx=4), dict(ldg=4),
    dict(ldg=-5), dict(x=None), dict(labels=None), dict(loss=None), dict(dx=P), dict(workspace=64), dict(workspace=0), dict(opts=False)])
def test_loss_refuses(kw):
    assert _loss(**kw) == BAD


def _adamw(count=1, opts=True, tensors=True, o=(), **kw):
    t = gnn.GnnAdamWTensor(param=256, grad=256, exp_avg=256, exp_avg_sq=256, n=10, state_bits=32)
    for k, v in kw.items():
        setattr(t, k, v)
    q = gnn.GnnAdamWOpts(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1)
    for k, v in dict(o).items():
        setattr(q, k, v)
    return gnn.load_library().gnn_adamw_step(ctypes.byref(t) if tensors else None, count, ctypes.byref(q) if opts else None)


@pytest.mark.parametrize("kw", [
    dict(count=-1), dict(opts=False), dict(tensors=False), dict(n=-1), dict(dtype=2), dict(state_bits=16), dict(state_bits=0), dict(weight_decay=-0.1),
    dict(weight_decay=float("nan")), dict(param=None), dict(exp_avg=None), dict(exp_avg_sq=None), dict(state_bits=8), dict(state_bits=8, scale=256),
    dict(master=256), dict(param=258), dict(grad=257), dict(exp_avg=258), dict(dtype=1, param=257), dict(state_bits=8, scale=258, scale_sq=256),
    dict(o=dict(step=0)), dict(o=dict(step=-3)), dict(o=dict(lr=-1.0)), dict(o=dict(lr=float("nan"))), dict(o=dict(beta1=1.0)), dict(o=dict(beta1=-0.1)),
    dict(o=dict(beta2=1.0)), dict(o=dict(beta2=float("nan"))), dict(o=dict(eps=-1e-8))])
def test_adamw_refuses(kw):
    assert _adamw(**kw) == BAD


def test_adamw_without_work_succeeds():
    assert _adamw(count=0, tensors=False) == OK
    assert _adamw(n=0, param=None, exp_avg=None, exp_avg_sq=None) == OK
    assert _adamw(grad=None) == OK  # left alone


def test_python_calls_refuse_host_tensors_and_wrong_types():
    x, v, s = torch.zeros(6, 4), torch.zeros(4), torch.zeros(1, 2)
    with pytest.raises(ValueError, match="device"):
        gnn.gnn_group_norm_fwd(x, v, v, x.clone(), s, s, 2, stream=0)
    with pytest.raises(TypeError):
        gnn.gnn_group_norm_fwd(x.double(), v, v, x.double(), s, s, 2, stream=0)
    with pytest.raises(ValueError, match="device"):
        gnn.gnn_softmax_xent(x, torch.zeros(6, dtype=torch.int32), torch.zeros(1), stream=0)
    with pytest.raises(TypeError):
        gnn.gnn_softmax_xent(x.half(), torch.zeros(6, dtype=torch.int32), torch.zeros(1), stream=0)
    with pytest.raises(ValueError, match="device"):
        gnn.AdamWTensors([v], [v], [v], [v])


@pytest.mark.gpu
def test_python_calls_refuse_wrong_shapes_and_types():
    dev = "cuda:0"
    x, y = torch.zeros(6, 4, device=dev), torch.zeros(6, 4, device=dev)
    v, s = torch.zeros(4, device=dev), torch.zeros(1, 2, device=dev)
    ws = torch.zeros(1 << 16, device=dev)
    ptr = torch.tensor([0, 6], device=dev)

    def norm(x=x, gamma=v, beta=v, y=y, mean=s, rstd=s, groups=2, workspace=ws, **kw):
        gnn.gnn_group_norm_fwd(x, gamma, beta, y, mean, rstd, groups, workspace=workspace, **kw)

    def norm_bwd(x=x, gamma=v, beta=v, mean=s, rstd=s, dy=torch.zeros_like(x), dx=y, dgamma=v, dbeta=v, groups=2, workspace=ws, **kw):
        gnn.gnn_group_norm_bwd(x, gamma, beta, mean, rstd, dy, dx, dgamma, dbeta, groups, workspace=workspace, **kw)
    norm()
    norm_bwd()
    for f, kw, error in (
            (norm, dict(y=y[:5]), ValueError), (norm, dict(y=y.bfloat16()), TypeError), (norm, dict(x=x.t().contiguous().t()), ValueError),
            (norm, dict(x=v), ValueError), (norm, dict(gamma=v[:3]), ValueError), (norm, dict(beta=v.double()), TypeError),
            (norm, dict(mean=s[:, :1]), ValueError), (norm, dict(rstd=torch.zeros(2, 2, device=dev)), ValueError), (norm, dict(groups=3), ValueError),
            (norm, dict(groups=0), ValueError), (norm, dict(workspace=None), gnn.GnnError), (norm, dict(workspace=ws[:2]), gnn.GnnError),
            (norm, dict(sample_ptr=ptr.float()), TypeError), (norm, dict(sample_ptr=ptr[:0]), ValueError), (norm, dict(sample_ptr=ptr[None]), ValueError),
            (norm, dict(sample_ptr=torch.tensor([0, 3, 6], device=dev)), ValueError), (norm, dict(n_samples=4), ValueError),
            (norm, dict(x=x[:1].expand(6, 4)), ValueError), (norm, dict(y=x), gnn.GnnError), (norm, dict(act=7), gnn.GnnError),
            (norm_bwd, dict(dy=y[:, :3]), ValueError), (norm_bwd, dict(dx=y.bfloat16()), TypeError), (norm_bwd, dict(dgamma=v[:2]), ValueError),
            (norm_bwd, dict(dx=x), gnn.GnnError), (norm_bwd, dict(dy=None), (TypeError, AttributeError))):
        with pytest.raises(error):
            f(**kw)
    t, loss = torch.zeros(6, dtype=torch.int32, device=dev), torch.zeros(1, device=dev)
    gnn.gnn_softmax_xent(x, t, loss, y, workspace=ws)
    for args, kw, error in (
            ((x, t[:5], loss, y), {}, ValueError), ((x, t.float(), loss, y), {}, TypeError), ((x, t, loss, y[:, :3]), {}, ValueError),
            ((x, t, loss.double(), y), {}, TypeError), ((x, t, v, y), {}, ValueError), ((x, t, loss, x), {}, gnn.GnnError),
            ((x, t, loss, y, v), {}, ValueError), ((x, t, loss, y), dict(reduction=4), gnn.GnnError), ((x, t[::2], loss, y), {}, ValueError)):
        with pytest.raises(error):
            gnn.gnn_softmax_xent(*args, workspace=ws, **kw)
    p = torch.zeros(300, device=dev)
    q, sc = torch.zeros(300, dtype=torch.uint8, device=dev), torch.zeros(2, device=dev)
    ok = dict(params=[p], grads=[p.clone()], exp_avg=[p.clone()], exp_avg_sq=[p.clone()])
    gnn.AdamWTensors(**ok)
    gnn.AdamWTensors(**{**ok, "exp_avg": [q], "exp_avg_sq": [q.clone()]}, scale=[sc], scale_sq=[sc.clone()])
    for kw, error in (
            (dict(grads=[p, p]), ValueError), (dict(grads=[p[:5]]), ValueError), (dict(grads=[p.bfloat16()]), TypeError), (dict(exp_avg=[q]), TypeError),
            (dict(exp_avg=[p.double()], exp_avg_sq=[p.double()]), TypeError), (dict(exp_avg=[q], exp_avg_sq=[q]), ValueError),
            (dict(exp_avg=[q], exp_avg_sq=[q], scale=[sc[:1]], scale_sq=[sc]), ValueError), (dict(master=[p.clone()]), TypeError),
            (dict(params=[p[::2]]), ValueError), (dict(weight_decay=[0.1, 0.2]), ValueError), (dict(params=[p.half()], grads=[p.half()]), TypeError)):
        with pytest.raises(error):
            gnn.AdamWTensors(**{**ok, **kw})
    with pytest.raises(gnn.GnnError):
        gnn.gnn_adamw_step(gnn.AdamWTensors(**ok), 0, 1e-3)
    with pytest.raises(ValueError):
        gnn.gnn_adamw_step(gnn.AdamWTensors(**ok), 1, 1e-3, grad_scale=p)
