"""What the training operators refuse, before anything touches a GPU: the C entry points of include/moe_spec_train.h with bad
sizes, types, strides, pointers and workspaces, and the torch layer with tensors it does not take."""
import ctypes as C

import pytest
import torch

from paper_2603_19289_amd import moe_spec as M
from paper_2603_19289_amd import training as T

ADDR = 1 << 20                                    # an address that is never followed: every call below is refused first


def refused(rc, *words):
    assert rc == M.EINVAL
    text = M.lib().moe_spec_train_last_error().decode()
    for w in words:
        assert w in text, text


def ln_forward(**kw):
    a = dict(stream=None, dtype=M.F32, x=ADDR, x_stride=64, rows=4, cols=64, gain=ADDR, bias=ADDR, eps=1e-5, y=ADDR * 2,
             y_stride=64, mean=ADDR, rstd=ADDR)
    a.update(kw)
    return M.lib().moe_spec_layernorm_forward(*a.values())


@pytest.mark.parametrize("bad,word", [(dict(dtype=2), "dtype"), (dict(rows=-1), "rows"), (dict(rows=1 << 31), "rows"), (dict(cols=0), "cols"),
                                      (dict(cols=8193), "cols"), (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"),
                                      (dict(x=None), "x is null"), (dict(x=ADDR + 2), "aligned"), (dict(y=None), "y is null"),
                                      (dict(y=ADDR + 1, dtype=M.BF16), "aligned"), (dict(y_stride=63), "stride"), (dict(x_stride=-64), "stride"),
                                      (dict(x_stride=1 << 40), "stride"), (dict(y=ADDR, x_stride=128), "in place"),
                                      (dict(gain=ADDR + 2), "gain"), (dict(rstd=ADDR + 1), "rstd")])
def test_layernorm_forward_refuses(bad, word):
    refused(ln_forward(**bad), "layernorm_forward", word)


def test_no_rows_need_no_pointers():
    assert ln_forward(rows=0, x=None, y=None) == M.OK


def ln_backward(**kw):
    a = dict(stream=None, dtype=M.F32, dy=ADDR, dy_stride=64, x=ADDR * 2, x_stride=64, rows=4000, cols=64, mean=ADDR, rstd=ADDR,
             gain=ADDR, dx=ADDR * 3, dx_stride=64, dgain=ADDR, dbias=ADDR, workspace=ADDR,
             workspace_bytes=M.moe_spec_layernorm_backward_workspace_bytes(4000, 64))
    a.update(kw)
    return M.lib().moe_spec_layernorm_backward(*a.values())


@pytest.mark.parametrize("bad,word", [(dict(dtype=-1), "dtype"), (dict(rows=-5), "rows"), (dict(cols=10000), "cols"), (dict(dy=None), "dy is null"),
                                      (dict(x=ADDR + 1), "x is not aligned"), (dict(dx_stride=8), "dx"), (dict(dx=ADDR), "dx must not"),
                                      (dict(dx=ADDR * 2), "dx must not"), (dict(mean=None), "mean"), (dict(rstd=None), "rstd"),
                                      (dict(workspace=None), "workspace"), (dict(workspace=ADDR + 8), "workspace"),
                                      (dict(workspace_bytes=8), "workspace"), (dict(dgain=ADDR + 2), "dgain")])
def test_layernorm_backward_refuses(bad, word):
    refused(ln_backward(**bad), "layernorm_backward", word)


def test_layernorm_backward_asked_for_nothing_does_nothing():
    assert ln_backward(dx=None, dgain=None, dbias=None, workspace=None, workspace_bytes=0) == M.OK


def test_workspace_sizes():
    size = M.moe_spec_layernorm_backward_workspace_bytes
    assert size(-1, 64) == size(4, 0) == size(4, 8193) == size(1 << 31, 64) == 0
    assert size(0, 64) == size(100, 64) == 0 < size(2000, 64) <= size(4000, 64) <= size(4000, 65)       # few rows need none
    assert M.moe_spec_distill_loss_workspace_bytes(4, 257) == M.moe_spec_distill_loss_workspace_bytes(-1, 8) == 0
    assert M.moe_spec_balance_loss_workspace_bytes(4, 8, 17) == M.moe_spec_balance_loss_workspace_bytes(4, 8, 0) == 0
    assert M.moe_spec_balance_loss_workspace_bytes(100000, 256, 16) > M.moe_spec_distill_loss_workspace_bytes(100000, 256) > 0
    assert M.moe_spec_balance_loss_workspace_bytes(1, 256, 16) == M.moe_spec_distill_loss_workspace_bytes(1, 256) == 0    # one workgroup


def distill(**kw):
    a = dict(stream=None, student_dtype=M.F32, student=ADDR, student_stride=32, teacher_dtype=M.BF16, teacher=ADDR * 2,
             teacher_stride=32, rows=100000, n_experts=32, temperature=1.0, valid=None, loss=ADDR, grad=ADDR * 3, grad_stride=32,
             workspace=ADDR, workspace_bytes=1 << 20)
    a.update(kw)
    return M.lib().moe_spec_distill_loss(*a.values())


@pytest.mark.parametrize("bad,word", [(dict(student_dtype=3), "dtype"), (dict(teacher_dtype=-1), "dtype"), (dict(rows=-1), "rows"),
                                      (dict(n_experts=0), "n_experts"), (dict(n_experts=257), "n_experts"), (dict(temperature=0.0), "temperature"),
                                      (dict(temperature=-1.0), "temperature"), (dict(temperature=float("inf")), "temperature"),
                                      (dict(temperature=float("nan")), "temperature"), (dict(temperature=1e-45), "temperature"), (dict(temperature=3.5e-39), "temperature"),
                                      (dict(student=None), "student is null"), (dict(teacher=ADDR + 1), "teacher is not aligned"),
                                      (dict(grad_stride=31), "grad"), (dict(grad=ADDR, grad_stride=64), "another stride"),
                                      (dict(grad=ADDR * 2), "teacher"), (dict(loss=None), "loss"), (dict(workspace=None), "workspace"),
                                      (dict(workspace=ADDR + 4), "workspace"), (dict(workspace_bytes=16), "workspace")])
def test_distill_loss_refuses(bad, word):
    refused(distill(**bad), "distill_loss", word)


def balance(**kw):
    a = dict(stream=None, dtype=M.F32, logits=ADDR, logits_stride=32, rows=100000, n_experts=32, ids=ADDR, ids_stride=4, top_k=4,
             coef=1.0, valid=None, loss=ADDR, counts=ADDR, grad=ADDR * 3, grad_stride=32, workspace=ADDR, workspace_bytes=1 << 20)
    a.update(kw)
    return M.lib().moe_spec_balance_loss(*a.values())


@pytest.mark.parametrize("bad,word", [(dict(dtype=2), "dtype"), (dict(rows=-1), "rows"), (dict(n_experts=300), "n_experts"), (dict(top_k=0), "top_k"),
                                      (dict(top_k=17), "top_k"), (dict(rows=(1 << 31) // 4), "rows * top_k"), (dict(coef=float("nan")), "coef"), (dict(coef=float("inf")), "coef"),
                                      (dict(logits=None), "logits is null"), (dict(ids=None), "ids is null"), (dict(ids=ADDR + 2), "ids is not aligned"),
                                      (dict(grad=ADDR, grad_stride=40), "another stride"), (dict(counts=None), "counts"), (dict(loss=ADDR + 1), "loss"),
                                      (dict(workspace_bytes=64), "workspace")])
def test_balance_loss_refuses(bad, word):
    refused(balance(**bad), "balance_loss", word)


def adamw(tensor=None, n=1, **kw):
    cfg = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, grad_scale=1.0, step=1, grad_dtype=M.F32,
               moments=M.MOMENTS_8BIT)
    cfg.update(kw)
    t = dict(p=ADDR, grad=ADDR, m=ADDR, v=ADDR, m_exp=ADDR, v_exp=ADDR, copy=ADDR, n=100)
    t.update(tensor or {})
    arr = (M.AdamWTensor * 1)(M.AdamWTensor(**t))
    return M.lib().moe_spec_adamw_step(None, arr if n else None, n, C.byref(M.AdamWConfig(**cfg)))


@pytest.mark.parametrize("bad,word", [(dict(moments=2), "moments"), (dict(grad_dtype=5), "grad_dtype"), (dict(beta1=1.0), "beta1"),
                                      (dict(beta2=-0.1), "beta2"), (dict(beta1=float("nan")), "beta1"), (dict(eps=-1.0), "eps"),
                                      (dict(lr=float("nan")), "lr"), (dict(weight_decay=-1.0), "weight_decay"), (dict(step=0), "step"),
                                      (dict(step_dev=ADDR + 4), "step_dev"), (dict(grad_scale_dev=ADDR + 1), "grad_scale_dev"), (dict(n=-1), "tensors"),
                                      (dict(n=65537), "tensors"), (dict(tensor=dict(n=-1)), "n is out"), (dict(tensor=dict(p=None)), "null"),
                                      (dict(tensor=dict(m_exp=None)), "null"), (dict(tensor=dict(p=ADDR + 2)), "aligned"),
                                      (dict(tensor=dict(copy=ADDR + 1)), "aligned"), (dict(tensor=dict(m=ADDR + 1), moments=M.MOMENTS_32BIT), "aligned")])
def test_adamw_step_refuses(bad, word):
    refused(adamw(**bad), "adamw_step", word)


def test_adamw_calls_that_are_refused_for_want_of_pointers():
    assert M.lib().moe_spec_adamw_step(None, None, 0, None) == M.EINVAL
    cfg = M.AdamWConfig(beta1=0.9, beta2=0.99, step=1)
    assert M.lib().moe_spec_adamw_step(None, None, 1, C.byref(cfg)) == M.EINVAL
    one = (M.AdamWTensor * 1)(M.AdamWTensor(m=ADDR, v=ADDR, m_exp=ADDR, v_exp=ADDR, n=5))
    out = (C.c_void_p * 1)(None)
    refused(M.lib().moe_spec_adamw_read_moments(None, one, 1, M.F32, out, None), "read_moments", "null")
    refused(M.lib().moe_spec_adamw_read_moments(None, one, 1, 9, out, None), "out_dtype")
    refused(M.lib().moe_spec_adamw_read_moments(None, one, 1, M.F32, (C.c_void_p * 1)(ADDR + 2), None), "aligned")


@pytest.mark.skipif(torch.cuda.is_available(), reason="meant for a machine without a GPU")
def test_without_a_gpu_the_calls_fail_loudly():
    assert ln_forward() == M.EHIP and ln_backward() == M.EHIP and distill() == M.EHIP and balance() == M.EHIP and adamw() == M.EHIP


def test_torch_layer_refuses_tensors_it_does_not_take():
    x = torch.zeros(4, 8)
    for call in (lambda: T.layernorm_forward(x), lambda: T.layernorm_backward(x, x, x[:, 0], x[:, 0]), lambda: T.distill_loss(x, x),
                 lambda: T.balance_loss(x, torch.zeros(4, 2, dtype=torch.int32)), lambda: T.AdamW([x], lr=1e-3)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):
        T.AdamW([], lr=1e-3)
    with pytest.raises(ValueError):
        T.AdamW([x], lr=1e-3, state="int4")


def test_the_header_is_c():
    """The declarations compile as C99 by themselves."""
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-fsyntax-only", "-x", "c", os.path.join(root, "include", "moe_spec_train.h")],
                          capture_output=True, text=True)
    assert done.returncode == 0, done.stderr


def test_the_reason_of_a_failure_is_the_calling_threads():
    import threading
    refused(ln_forward(cols=0), "cols")
    seen = []

    def other():
        seen.append(M.lib().moe_spec_train_last_error())
        refused(distill(temperature=-1.0), "temperature")
    t = threading.Thread(target=other)
    t.start()
    t.join()
    assert seen == [b""] and b"cols" in M.lib().moe_spec_train_last_error()


MOST = (2 ** 24 - 1) * 2048                       # elements of an AdamW tensor: a launch has fewer than 2^32 threads, 256 a workgroup


@pytest.mark.parametrize("n", [MOST + 1, 1 << 35, 1 << 40])
def test_adamw_refuses_a_tensor_that_no_launch_can_take(n):
    refused(adamw(tensor=dict(n=n)), "adamw_step", "n is out")
    arr = (M.AdamWTensor * 2)(M.AdamWTensor(n=5, m=ADDR, m_exp=ADDR), M.AdamWTensor(n=n, m=ADDR, m_exp=ADDR))
    refused(M.lib().moe_spec_adamw_read_moments(None, arr, 2, M.BF16, (C.c_void_p * 2)(ADDR, ADDR), None), "read_moments", "n is out")


@pytest.mark.skipif(torch.cuda.is_available(), reason="meant for a machine without a GPU")
def test_adamw_takes_the_longest_tensor_that_it_names():
    assert adamw(tensor=dict(n=MOST)) == M.EHIP
