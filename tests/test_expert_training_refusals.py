"""What the operators that train a layer's experts refuse, before anything touches a GPU."""
import ctypes as C

import pytest
import torch

from paper_2603_19289_amd import moe_spec as M
from paper_2603_19289_amd import training as T

ADDR = 1 << 20                                    # an address that is never followed: every call below is refused first
NAN, INF = float("nan"), float("inf")


def refused(rc, *words):
    assert rc == M.EINVAL
    text = M.lib().moe_spec_train_last_error().decode()
    for w in words:
        assert w in text, text


def product(**kw):
    a = dict(stream=None, dtype=M.F32, x=ADDR, x_stride=64, rows=40, w=ADDR * 2, w_stride=64, w_expert_stride=32 * 64, n_experts=4, n=32, k=64,
             ends=ADDR, transpose=0, out_dtype=M.F32, y=ADDR * 3, y_stride=32)
    a.update(kw)
    return M.lib().moe_spec_grouped_product(*a.values())


@pytest.mark.parametrize("bad,word", [(dict(dtype=2), "dtype"), (dict(out_dtype=-1), "out_dtype"), (dict(rows=-1), "rows"), (dict(rows=1 << 31), "rows"),
                                      (dict(n_experts=0), "n_experts"), (dict(n_experts=257), "n_experts"), (dict(n=0), "n and k"), (dict(k=65537), "n and k"),
                                      (dict(x=None), "x is null"), (dict(x=ADDR + 2), "x is not aligned"), (dict(x_stride=-1), "x has"), (dict(w=None), "w is null"),
                                      (dict(w_stride=-64), "w has"), (dict(w_expert_stride=-1), "w_expert_stride"), (dict(w_expert_stride=(1 << 40) + 1), "w_expert_stride"),
                                      (dict(y=None), "y is null"), (dict(y_stride=31), "y has"), (dict(transpose=1, y_stride=63), "y has"), (dict(y=ADDR), "y must not"),
                                      (dict(y=ADDR * 2), "y must not"), (dict(ends=None), "ends"), (dict(ends=ADDR + 2), "ends")])
def test_grouped_product_refuses(bad, word):
    refused(product(**bad), "grouped_product", word)


def weight_grad(**kw):
    a = dict(stream=None, dtype=M.BF16, dy=ADDR, dy_stride=32, x=ADDR * 2, x_stride=64, rows=40, n_experts=4, n=32, k=64, ends=ADDR, out_dtype=M.F32,
             dw=ADDR * 3, dw_stride=64, dw_expert_stride=32 * 64, workspace=ADDR, workspace_bytes=1 << 30)
    a.update(kw)
    return M.lib().moe_spec_grouped_weight_grad(*a.values())


@pytest.mark.parametrize("bad,word", [(dict(dtype=3), "dtype"), (dict(out_dtype=2), "out_dtype"), (dict(rows=-1), "rows"), (dict(n_experts=300), "n_experts"),
                                      (dict(n=65537), "n and k"), (dict(k=0), "n and k"), (dict(dy=None), "dy is null"), (dict(dy=ADDR + 1), "dy is not aligned"),
                                      (dict(x=None), "x is null"), (dict(x_stride=-1), "x has"), (dict(dw=None), "dw is null"), (dict(dw=ADDR * 3 + 2), "dw is not aligned"),
                                      (dict(dw_stride=63), "dw has"), (dict(dw_expert_stride=32 * 64 - 1), "dw_expert_stride"), (dict(dw=ADDR), "dw must not"),
                                      (dict(ends=None), "ends"), (dict(rows=4000, workspace=None), "workspace"), (dict(rows=4000, workspace=ADDR + 8), "workspace"),
                                      (dict(rows=4000, workspace_bytes=8), "workspace")])
def test_grouped_weight_grad_refuses(bad, word):
    refused(weight_grad(**bad), "grouped_weight_grad", word)


def test_weight_grad_workspace():
    size = M.moe_spec_grouped_weight_grad_workspace_bytes
    for dtype in (M.F32, M.BF16):
        assert size(dtype, -1, 4, 8, 8) == size(dtype, 4, 0, 8, 8) == size(dtype, 4, 257, 8, 8) == size(dtype, 4, 1, 0, 8) == size(dtype, 4, 1, 8, 65537) == 0
        assert size(dtype, 0, 4, 32, 64) == size(dtype, 700, 4, 32, 64) == 0 and size(dtype, 100000, 128, 1536, 2048) == 0
        assert size(dtype, 20000, 4, 32, 64) % (4 * 32 * 64 * 4) == 0 < size(dtype, 20000, 4, 32, 64) <= 64 * 4 * 32 * 64 * 4
        assert weight_grad(dtype=dtype, dy=ADDR * 4, x=ADDR * 5, dw_stride=64, workspace=None, workspace_bytes=0, rows=-1) == M.EINVAL
    assert size(7, 100000, 4, 32, 64) == 0


def test_too_large_for_a_launch():
    refused(product(rows=(1 << 31) - 1, n=65536, y_stride=65536), "grouped_product", "one launch")


def forward(**kw):
    a = dict(stream=None, dtype=M.F32, a=ADDR, a_stride=128, rows=4, cols=64, weight=ADDR, h=ADDR * 2, h_stride=64)
    a.update(kw)
    return M.lib().moe_spec_swiglu_forward(*a.values())


def backward(**kw):
    a = dict(stream=None, dtype=M.F32, dh=ADDR, dh_stride=64, a=ADDR * 2, a_stride=128, rows=4, cols=64, weight=ADDR, da=ADDR * 3, da_stride=128, dweight=ADDR)
    a.update(kw)
    return M.lib().moe_spec_swiglu_backward(*a.values())


@pytest.mark.parametrize("bad,word", [(dict(dtype=2), "dtype"), (dict(rows=-1), "rows"), (dict(rows=1 << 31), "rows"), (dict(cols=0), "cols"), (dict(cols=65537), "cols"),
                                      (dict(a=None), "a is null"), (dict(a=ADDR * 4 + 1), "a is not aligned"), (dict(a_stride=-2), "a has"), (dict(weight=ADDR + 1), "weight")])
def test_swiglu_refuses(bad, word):
    refused(forward(**bad), "swiglu_forward", word)
    refused(backward(**bad), "swiglu_backward", word)


def test_swiglu_refuses_outputs():
    refused(forward(h=None), "h is null")
    refused(forward(h_stride=63), "h has")
    refused(forward(h=ADDR), "h must not")
    refused(backward(da_stride=127), "da has")
    refused(backward(da=ADDR), "da must not")
    refused(backward(da=ADDR * 2), "da must not")
    refused(backward(dh=None), "dh is null")
    refused(backward(dweight=ADDR + 2), "dweight")


def orthogonalise(**kw):
    a = dict(stream=None, dtype=M.F32, g=ADDR, g_matrix_stride=80 * 96, g_stride=96, count=3, rows=80, cols=96, coefficients=(C.c_double * 3)(1.5, -0.5, 0.0),
             iterations=5, out=ADDR * 2, out_matrix_stride=80 * 96, out_stride=96, workspace=ADDR, workspace_bytes=1 << 30)
    a.update(kw)
    return M.lib().moe_spec_orthogonalise(*a.values())


@pytest.mark.parametrize("bad,word", [(dict(dtype=2), "dtype"), (dict(count=-1), "negative"), (dict(rows=-1), "negative"), (dict(cols=65537), "65536"),
                                      (dict(count=1 << 40), "2^32"), (dict(count=1 << 30, rows=1, cols=1, g_matrix_stride=1, out_matrix_stride=1), "one launch"), (dict(coefficients=None), "coefficients"), (dict(coefficients=(C.c_double * 3)(NAN, 0, 0)), "coefficients"),
                                      (dict(coefficients=(C.c_double * 3)(1, INF, 0)), "coefficients"), (dict(coefficients=(C.c_double * 3)(1, 0, -17)), "coefficients"),
                                      (dict(iterations=0), "iterations"), (dict(iterations=65), "iterations"), (dict(g=None), "g is null"), (dict(g=ADDR + 1), "g is not"),
                                      (dict(g_stride=-1), "g has"), (dict(g_matrix_stride=-1), "g's matrix"), (dict(out=None), "out is null"), (dict(out=ADDR + 1), "out is not"),
                                      (dict(out_stride=95), "out has"), (dict(out_matrix_stride=100), "out's matrix"), (dict(out=ADDR), "out must not"),
                                      (dict(workspace=None), "workspace"), (dict(workspace=ADDR + 8), "workspace"), (dict(workspace_bytes=1000), "workspace")])
def test_orthogonalise_refuses(bad, word):
    refused(orthogonalise(**bad), "orthogonalise", word)


def muon(tensor=None, n=1, workspace=ADDR, workspace_bytes=1 << 30, null=False, **kw):
    cfg = dict(lr=1e-3, momentum=0.9, weight_decay=0.0, update_rms=0.2, grad_scale=1.0, coefficients=(3.4445, -4.775, 2.0315), iterations=5, nesterov=1,
               grad_dtype=M.F32)
    cfg.update(kw)
    t = dict(p=ADDR, grad=ADDR, m=ADDR, copy=ADDR, count=2, rows=160, cols=240)
    t.update(tensor or {})
    return M.lib().moe_spec_muon_step(None, None if null else (M.MuonTensor * 1)(M.MuonTensor(**t)), n, C.byref(M.MuonConfig(**cfg)), workspace, workspace_bytes)


@pytest.mark.parametrize("bad,word", [(dict(grad_dtype=4), "grad_dtype"), (dict(momentum=1.0), "momentum"), (dict(momentum=-0.1), "momentum"), (dict(momentum=NAN), "momentum"),
                                      (dict(lr=NAN), "lr"), (dict(weight_decay=-1.0), "weight_decay"), (dict(update_rms=-1.0), "update_rms"), (dict(update_rms=NAN), "update_rms"),
                                      (dict(iterations=0), "iterations"), (dict(coefficients=(NAN, 0, 0)), "coefficients"), (dict(grad_scale_dev=ADDR + 1), "grad_scale_dev"),
                                      (dict(n=-1), "tensors"), (dict(n=65537), "tensors"), (dict(null=True), "tensors"), (dict(tensor=dict(count=-1)), "negative"),
                                      (dict(tensor=dict(rows=70000)), "65536"), (dict(tensor=dict(p=None)), "null"), (dict(tensor=dict(grad=None)), "null"), (dict(tensor=dict(m=None)), "null"),
                                      (dict(tensor=dict(copy=ADDR + 1)), "aligned"), (dict(tensor=dict(copy_stride=160 * 240 - 1)), "copy_stride"), (dict(tensor=dict(copy_stride=-1)), "copy_stride"), (dict(tensor=dict(m=ADDR + 2)), "aligned"), (dict(workspace=None), "workspace"),
                                      (dict(workspace=ADDR + 4), "workspace"), (dict(workspace_bytes=64), "workspace")])
def test_muon_step_refuses(bad, word):
    refused(muon(**bad), "muon_step", word)


def test_sizes_without_work_need_nothing():
    assert product(rows=0, x=None, w=None, y=None) == M.OK
    assert forward(rows=0, a=None, h=None) == M.OK and backward(rows=0, a=None, dh=None, da=None) == M.OK
    assert orthogonalise(count=0, g=None, out=None, workspace=None) == M.OK and orthogonalise(rows=0, g=None, out=None, workspace=None) == M.OK
    assert muon(tensor=dict(count=0, p=None), workspace=None, workspace_bytes=0) == M.OK and muon(n=0, null=True, workspace=None) == M.OK
    assert M.moe_spec_orthogonalise_workspace_bytes(0, 5, 5) == M.moe_spec_orthogonalise_workspace_bytes(1, 70000, 5) == 0
    assert M.moe_spec_orthogonalise_workspace_bytes(2, 500, 5000) > M.moe_spec_orthogonalise_workspace_bytes(1, 500, 5000) > 0
    assert M.moe_spec_orthogonalise_workspace_bytes(20, 5, 5) == 0 < M.moe_spec_orthogonalise_workspace_bytes(1, 65, 65)      # small ones need none
    assert M.lib().moe_spec_muon_step(None, None, 0, None, None, 0) == M.EINVAL


@pytest.mark.skipif(torch.cuda.is_available(), reason="meant for a machine without a GPU")
def test_without_a_gpu_the_calls_fail_loudly():
    assert [f() for f in (product, weight_grad, forward, backward, orthogonalise, muon)] == [M.EHIP] * 6


def test_torch_layer_refuses_tensors_it_does_not_take():
    x, w, ends = torch.zeros(4, 8), torch.zeros(2, 6, 8), torch.zeros(2, dtype=torch.int32)
    for call in (lambda: T.grouped_product(x, w, ends), lambda: T.grouped_weight_grad(x, x, ends), lambda: T.swiglu_forward(x), lambda: T.swiglu_backward(x, x),
                 lambda: T.orthogonalise(x), lambda: T.Muon([x], lr=0.1), lambda: T.Muon([], lr=0.1)):
        with pytest.raises(ValueError):
            call()


@pytest.fixture
def recorded(monkeypatch):
    """Calls into the library are recorded instead of made, and tensors of the CPU are taken."""
    made = []
    monkeypatch.setattr(T, "_queue", lambda dev, call, *args: made.append(args))
    monkeypatch.setattr(T, "_rows", lambda t, name, like=None: T._TYPES[t.dtype])
    monkeypatch.setattr(T.Muon, "_tensor", lambda self, t, name, dtype, shape: None)
    return made


def test_torch_layer_checks_shapes_and_types(recorded):
    x, w, ends = torch.zeros(4, 8), torch.zeros(2, 6, 8), torch.zeros(2, dtype=torch.int32)
    T.grouped_product(x, w, ends)
    assert recorded[-1][2:4] == (8, 4) and recorded[-1][5:10] == (8, 48, 2, 6, 8)
    bad = [dict(x=torch.zeros(4, 6)), dict(transpose=True), dict(w=w[0]), dict(w=w.bfloat16()), dict(w=w.transpose(1, 2)), dict(ends=ends[:1]), dict(ends=ends.long()),
           dict(dtype=torch.float16), dict(out=torch.zeros(4, 7)), dict(out=torch.zeros(4, 6, dtype=torch.bfloat16)), dict(out=torch.zeros(6, 4).t()),
           dict(w=torch.zeros(257, 6, 8), ends=torch.zeros(257, dtype=torch.int32)), dict(w=torch.zeros(0, 6, 8), ends=ends[:0]),
           dict(out=torch.zeros(4, 6, requires_grad=True))]
    for kw in bad:
        with pytest.raises(ValueError):
            T.grouped_product(**dict(dict(x=x, w=w, ends=ends), **kw))
    for kw in (dict(dy=torch.zeros(5, 6)), dict(dy=torch.zeros(4, 6).bfloat16()), dict(ends=ends.float()), dict(dtype=torch.int32), dict(out=torch.zeros(2, 8, 6)),
               dict(out=torch.zeros(2, 6, 8, requires_grad=True))):
        with pytest.raises(ValueError):
            T.grouped_weight_grad(**dict(dict(dy=torch.zeros(4, 6), x=x, ends=ends), **kw))
    for call in (lambda: T.swiglu_forward(torch.zeros(4, 7)), lambda: T.swiglu_forward(x, torch.zeros(5)), lambda: T.swiglu_forward(x, torch.zeros(4).double()),
                 lambda: T.swiglu_backward(x, x), lambda: T.swiglu_backward(torch.zeros(4, 4).bfloat16(), x), lambda: T.swiglu_forward(torch.zeros(4, 0))):
        with pytest.raises(ValueError):
            call()


def test_muon_follows_tensors_that_get_other_storage(recorded):
    p = [torch.zeros(3, 4, 5), torch.zeros(6, 7)]
    opt = T.Muon(p, lr=0.1, copies=[None, torch.zeros(6, 7, dtype=torch.bfloat16)])
    g = [torch.zeros(3, 4, 5), torch.zeros(6, 7)]

    def table():
        return [(d.p, d.grad, d.m, d.copy, d.count, d.rows, d.cols) for d in opt._desc]
    before = []
    for t in (None, p[0], p[1], opt.copies[1], opt.states()["m"][0], opt.states()["m"][1]):
        if t is not None:
            before.append(t.data)
            t.data = t.data.clone()
        opt.step(g)
        m = opt.states()["m"]
        assert table() == [(p[0].data_ptr(), g[0].data_ptr(), m[0].data_ptr(), None, 3, 4, 5),
                           (p[1].data_ptr(), g[1].data_ptr(), m[1].data_ptr(), opt.copies[1].data_ptr(), 1, 6, 7)]
    blocks = torch.zeros(3, 50, dtype=torch.bfloat16)
    other = T.Muon([torch.zeros(3, 4, 5)], lr=0.1, copies=[blocks[:, 10:30].unflatten(1, (4, 5))])
    assert other._desc[0].copy == blocks.data_ptr() + 20 and other._desc[0].copy_stride == 50
    opt.step([None, g[1]])
    assert [d[4] for d in table()] == [0, 1]
    p[0].data = opt.states()["m"][0].data
    with pytest.raises(ValueError):
        opt.step(g)
    for bad in (lambda: T.Muon([torch.zeros(5)], lr=0.1), lambda: T.Muon(p, lr=0.1, copies=[None]), lambda: T.Muon([g[1], g[1]], lr=0.1),
                lambda: T.Muon([g[1]], lr=0.1, states={"m": []}), lambda: T.Muon([g[1]], lr=0.1).step([]), lambda: T.Muon([g[1]], lr=0.1).step([g[1].double()])):
        with pytest.raises(ValueError):
            bad()
