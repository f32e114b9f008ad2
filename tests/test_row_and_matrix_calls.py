"""Refusals of the calls on rows by id and on weight matrices: the C entry points return before any device work, the Python calls raise."""
import ctypes

import pytest
import torch

import paper_2104_06700_amd as gnn

BAD, OK = gnn.GNN_ERR_INVALID_ARG, gnn.GNN_OK
P, Q, IDS = 256, 512, 1024  # never dereferenced: every call below returns before touching memory


def test_struct_layouts_match_the_header():
    # gnn_lookup_opts: 4 x int32, float, int32, 2 x int64, 2 pointers, int64; gnn_store_opts: 4 x int32, 2 x int64, 2 pointers, int64
    assert ctypes.sizeof(gnn.GnnLookupOpts) == 24 + 16 + 24
    assert ctypes.sizeof(gnn.GnnStoreOpts) == 16 + 16 + 24
    # gnn_orthogonalize_matrix: 2 pointers, 4 x int64, 2 x int32; its options: 4 doubles, 2 x int32, 2 pointers, int64
    assert ctypes.sizeof(gnn.GnnOrthogonalizeMatrix) == 16 + 32 + 8
    assert ctypes.sizeof(gnn.GnnOrthogonalizeOpts) == 32 + 8 + 24
    # gnn_muon_matrix: 4 pointers, 2 x int64, int32, 2 floats, int32; its options: 6 doubles, 2 x int32, 3 pointers, int64
    assert ctypes.sizeof(gnn.GnnMuonMatrix) == 32 + 16 + 16
    assert ctypes.sizeof(gnn.GnnMuonOpts) == 48 + 8 + 32


def _lookup(backward=False, table=P, ids=IDS, y=Q, v=100, n=50, f=16, opts=True, workspace=4096, room=1 << 30, **kw):
    o = gnn.GnnLookupOpts(scale=1.0, workspace=workspace, workspace_bytes=room)
    for k, x in kw.items():
        setattr(o, k, x)
    lib = gnn.load_library()
    o = ctypes.byref(o) if opts else None
    return lib.gnn_lookup_bwd(ids, y, table, v, n, f, o) if backward else lib.gnn_lookup_fwd(table, ids, y, v, n, f, o)


@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("kw", [
    dict(v=-1), dict(n=-1), dict(f=-1), dict(v=1 << 31), dict(n=1 << 31), dict(f=(1 << 24) + 1), dict(table_dtype=2), dict(dtype=-1), dict(ids_is_64=2),
    dict(accumulate=2), dict(ldt=15), dict(ldy=15), dict(ldt=-16), dict(table=None), dict(ids=None), dict(y=None), dict(y=P), dict(table=P + 2),
    dict(y=Q + 1), dict(dtype=1, y=Q + 1), dict(ids=IDS + 2), dict(ids_is_64=1, ids=IDS + 4), dict(opts=False)])
def test_lookup_refuses(kw, backward):
    assert _lookup(backward, **kw) == BAD


def test_lookup_workspace_and_empty_calls():
    assert _lookup(True, workspace=None) == BAD and _lookup(True, workspace=4100) == BAD and _lookup(True, room=100) == BAD
    assert _lookup(n=0, ids=None, y=None) == OK and _lookup(f=0) == OK
    assert _lookup(True, v=0, table=None) == OK and _lookup(True, f=0) == OK and _lookup(True, n=0, ids=None, y=None, accumulate=1) == OK
    size = gnn.gnn_lookup_workspace_bytes
    assert size(0, 10, 10) == size(10, 0, 10) == size(10, 10, 0) == size(-1, 10, 10) == size(1 << 31, 1, 1) == 0
    assert size(100, 1000, 16) >= 4 * 1000 * 4
    assert _lookup(True, room=size(100, 50, 16) - 1) == BAD


def _store(read=False, x=P, ids=IDS, store=Q, v=100, n=50, f=40, opts=True, workspace=4096, room=1 << 30, **kw):
    o = gnn.GnnStoreOpts(workspace=workspace, workspace_bytes=room)
    for k, t in kw.items():
        setattr(o, k, t)
    lib = gnn.load_library()
    o = ctypes.byref(o) if opts else None
    return lib.gnn_load_rows(store, ids, x, v, n, f, o) if read else lib.gnn_store_rows(x, ids, store, v, n, f, o)


@pytest.mark.parametrize("read", [False, True])
@pytest.mark.parametrize("kw", [
    dict(v=-1), dict(n=-1), dict(f=-1), dict(v=1 << 31), dict(n=1 << 31), dict(f=(1 << 24) + 1), dict(dtype=2), dict(ids_is_64=-1), dict(unique=2),
    dict(lds=41), dict(lds=-48), dict(ldx=39), dict(x=None), dict(store=None), dict(store=P), dict(ids=None, n=101), dict(x=P + 2), dict(dtype=1, x=P + 1),
    dict(ids=IDS + 2), dict(ids_is_64=1, ids=IDS + 4), dict(opts=False)])
def test_store_refuses(kw, read):
    assert _store(read, **kw) == BAD


def test_store_sizes_workspace_and_empty_calls():
    assert [gnn.gnn_store_row_bytes(f) for f in (-1, 0, 1, 15, 16, 31, 32, 33, 100, 256)] == [0, 0, 16, 16, 32, 32, 48, 48, 112, 272]
    assert gnn.gnn_store_rows_workspace_bytes(1000, 100) == 0 and gnn.gnn_store_rows_workspace_bytes(1000, 1 << 20) == 4000
    assert gnn.gnn_store_rows_workspace_bytes(-1, 1 << 20) == gnn.gnn_store_rows_workspace_bytes(1000, -1) == 0
    assert _store(n=0, x=None) == OK and _store(f=0) == OK and _store(v=0, store=None) == OK and _store(True, n=0, x=None) == OK
    assert _store(v=1000, n=5000, workspace=None) == BAD and _store(v=1000, n=5000, room=3999) == BAD and _store(v=1000, n=5000, workspace=4098) == BAD


def _orthogonalize(count=1, opts=True, matrices=True, o=(), **kw):
    t = gnn.GnnOrthogonalizeMatrix(in_=P, out=Q, rows=10, cols=20)
    for k, x in kw.items():
        setattr(t, k, x)
    q = gnn.GnnOrthogonalizeOpts(a=1.5, b=-0.5, c=0.0, eps=1e-7, steps=5, workspace=4096, workspace_bytes=1 << 30)
    for k, x in dict(o).items():
        setattr(q, k, x)
    return gnn.load_library().gnn_orthogonalize(ctypes.byref(t) if matrices else None, count, ctypes.byref(q) if opts else None)


@pytest.mark.parametrize("kw", [
    dict(count=-1), dict(matrices=False), dict(opts=False), dict(rows=-1), dict(cols=65537), dict(dtype=2), dict(ld_in=19), dict(ld_out=-20), dict(in_=None),
    dict(out=None), dict(in_=P + 2), dict(out=Q + 1), dict(dtype=1, in_=P + 1), dict(out=P, ld_in=20, ld_out=24), dict(o=dict(steps=0)), dict(o=dict(steps=101)),
    dict(o=dict(eps=0.0)), dict(o=dict(eps=float("nan"))), dict(o=dict(a=float("inf"))), dict(o=dict(b=float("nan"))), dict(o=dict(c=float("inf"))),
    dict(o=dict(workspace=None)), dict(o=dict(workspace=4112)), dict(o=dict(workspace_bytes=1000))])
def test_orthogonalize_refuses(kw):
    assert _orthogonalize(**kw) == BAD


def _muon(count=1, opts=True, matrices=True, o=(), **kw):
    t = gnn.GnnMuonMatrix(param=P, grad=Q, momentum=IDS, rows=10, cols=20, update_scale=1.0)
    for k, x in kw.items():
        setattr(t, k, x)
    q = gnn.GnnMuonOpts(lr=0.02, momentum=0.9, a=1.5, b=-0.5, c=0.0, eps=1e-7, nesterov=1, steps=5, workspace=4096, workspace_bytes=1 << 30)
    for k, x in dict(o).items():
        setattr(q, k, x)
    return gnn.load_library().gnn_muon_step(ctypes.byref(t) if matrices else None, count, ctypes.byref(q) if opts else None)


@pytest.mark.parametrize("kw", [
    dict(count=-1), dict(matrices=False), dict(opts=False), dict(rows=-1), dict(rows=65537), dict(dtype=-1), dict(weight_decay=-0.1),
    dict(weight_decay=float("nan")), dict(update_scale=float("inf")), dict(param=None), dict(momentum=None), dict(master=P), dict(param=P + 2), dict(grad=Q + 2),
    dict(momentum=IDS + 2), dict(dtype=1, master=P + 2), dict(o=dict(lr=-1.0)), dict(o=dict(lr=float("inf"))), dict(o=dict(momentum=1.0)), dict(o=dict(momentum=-0.1)),
    dict(o=dict(nesterov=2)), dict(o=dict(steps=0)), dict(o=dict(eps=-1.0)), dict(o=dict(a=float("nan"))), dict(o=dict(workspace=None)),
    dict(o=dict(workspace=4100)), dict(o=dict(workspace_bytes=1000))])
def test_muon_refuses(kw):
    assert _muon(**kw) == BAD


def test_matrices_without_work():
    assert _orthogonalize(count=0, matrices=False, o=dict(workspace=None)) == OK and _orthogonalize(rows=0, in_=None, out=None, o=dict(workspace=None)) == OK
    assert _muon(count=0, matrices=False, o=dict(workspace=None)) == OK and _muon(cols=0, param=None, o=dict(workspace=None)) == OK
    assert _muon(grad=None, o=dict(workspace=None)) == OK  # left alone
    lib = gnn.load_library()
    t = gnn.GnnOrthogonalizeMatrix(in_=P, out=Q, rows=100, cols=200)
    assert lib.gnn_orthogonalize_workspace_bytes(ctypes.byref(t), 1) >= 6 * (3 * 100 * 200 + 2 * 100 * 100)
    assert lib.gnn_orthogonalize_workspace_bytes(None, 1) == 0 and lib.gnn_orthogonalize_workspace_bytes(ctypes.byref(t), -1) == 0
    t.rows = -1
    assert lib.gnn_orthogonalize_workspace_bytes(ctypes.byref(t), 1) == 0
    # the largest there is does not overflow
    t.rows = t.cols = 65536
    assert lib.gnn_orthogonalize_workspace_bytes(ctypes.byref(t), 1) >= 30 * 65536 * 65536


def test_python_calls_refuse_host_tensors_and_wrong_types():
    x, ids, store = torch.zeros(6, 4), torch.zeros(6, dtype=torch.int32), torch.zeros(6, 16, dtype=torch.uint8)
    with pytest.raises(ValueError, match="device"):
        gnn.gnn_lookup_fwd(x, ids, x.clone(), stream=0)
    with pytest.raises(TypeError):
        gnn.gnn_lookup_fwd(x.double(), ids, x, stream=0)
    with pytest.raises(ValueError, match="device"):
        gnn.gnn_lookup_bwd(ids, x, x.clone(), stream=0)
    with pytest.raises(ValueError, match="device"):
        gnn.gnn_store_rows(x, store, ids, stream=0)
    with pytest.raises(TypeError):
        gnn.gnn_store_rows(x.half(), store, ids, stream=0)
    for make in (lambda: gnn.OrthogonalizeTensors([x], [x]), lambda: gnn.MuonTensors([x], [x], [x])):
        with pytest.raises(ValueError, match="device"):
            make()


@pytest.mark.gpu
def test_python_calls_refuse_wrong_shapes_and_types():
    dev = "cuda:0"
    table, y, ids = torch.zeros(9, 4, device=dev), torch.zeros(6, 4, device=dev), torch.zeros(6, dtype=torch.int32, device=dev)
    ws = torch.zeros(1 << 16, device=dev)
    gnn.gnn_lookup_fwd(table, ids, y)
    for args, error in (((table, ids[:5], y), ValueError), ((table, ids.float(), y), TypeError), ((table, ids[None], y), ValueError),
                        ((table, ids, y[:, :3]), ValueError), ((table.half(), ids, y), TypeError), ((table, ids[::2], y[:3]), ValueError),
                        ((table, ids, y.t().contiguous().t()), ValueError), ((table[0], ids, y), ValueError), ((table, None, y), (TypeError, AttributeError)),
                        ((table, ids, table[:6]), gnn.GnnError)):
        with pytest.raises(error):
            gnn.gnn_lookup_fwd(*args)
    gnn.gnn_lookup_bwd(ids, y, table, workspace=ws)
    for args, kw, error in (((ids[:5], y, table), {}, ValueError), ((ids, y, table[:, :3]), {}, ValueError), ((ids, y, table), dict(workspace=None), gnn.GnnError),
                            ((ids, y, table), dict(workspace=ws[:3]), gnn.GnnError), ((ids, y, table.double()), {}, TypeError)):
        with pytest.raises(error):
            gnn.gnn_lookup_bwd(*args, **{"workspace": ws, **kw})
    store = torch.zeros(9, 16, dtype=torch.uint8, device=dev)
    gnn.gnn_store_rows(y, store, ids)
    gnn.gnn_load_rows(store, y, ids)
    for args, error in (((y, store.float(), ids), TypeError), ((y, store[:, :4], ids), ValueError), ((y, store[:, ::2], ids), ValueError), ((y, store, ids[:3]), ValueError),
                        ((y, store[:5], None), gnn.GnnError), ((y, store[0], ids), ValueError), ((y, store[:1].expand(9, 16), ids), ValueError)):
        with pytest.raises(error):
            gnn.gnn_store_rows(*args)
        with pytest.raises(error):
            gnn.gnn_load_rows(args[1], args[0], args[2])
    p = torch.zeros(8, 12, device=dev)
    for ins, outs, error in (([p], [], ValueError), ([p], [p[:, :5]], ValueError), ([p], [p.bfloat16()], TypeError), ([p[0]], [p[0]], ValueError),
                             ([p.t()], [p.t()], ValueError), ([p.half()], [p.half()], TypeError)):
        with pytest.raises(error):
            gnn.OrthogonalizeTensors(ins, outs)
    with pytest.raises(gnn.GnnError):
        gnn.gnn_orthogonalize(gnn.OrthogonalizeTensors([p], [p]))
    with pytest.raises(ValueError):
        gnn.gnn_orthogonalize(gnn.OrthogonalizeTensors([p], [p]), coefficients=(1.0, 2.0), workspace=ws)
    ok = dict(params=[p], grads=[p.clone()], momentum=[p.clone()])
    gnn.gnn_muon_step(gnn.MuonTensors(**ok), 0.1, workspace=ws)
    for kw, error in ((dict(grads=[p, p]), ValueError), (dict(grads=[p[:5]]), ValueError), (dict(grads=[p.bfloat16()]), TypeError), (dict(momentum=[p.bfloat16()]), TypeError),
                      (dict(momentum=[p[:, :6].contiguous()]), ValueError), (dict(master=[p.clone()]), TypeError), (dict(params=[p[:, ::2]]), ValueError),
                      (dict(weight_decay=[0.1, 0.2]), ValueError), (dict(update_scale=[1.0, 2.0]), ValueError), (dict(params=[p.view(-1)]), ValueError),
                      (dict(params=[p.half()], grads=[p.half()]), TypeError)):
        with pytest.raises(error):
            gnn.MuonTensors(**{**ok, **kw})
    with pytest.raises(gnn.GnnError):
        gnn.gnn_muon_step(gnn.MuonTensors(**ok), -0.1, workspace=ws)
    with pytest.raises(gnn.GnnError):
        gnn.gnn_muon_step(gnn.MuonTensors(**ok), 0.1)
