"""What training.py does on the host, on a machine without a GPU: calls into the library are recorded instead of made, and the checks that
tensors lie on a GPU are left out."""
import pytest
import torch

from paper_2603_19289_amd import moe_spec as M
from paper_2603_19289_amd import training as T


@pytest.fixture
def calls(monkeypatch):
    """AdamW's tables as each call would hand them to the library: a list of tensors' addresses per call."""
    made = []

    def record(dev, call, desc, n, *rest):
        made.append([{k: getattr(d, k) for k, _ in M.AdamWTensor._fields_} for d in desc])
    monkeypatch.setattr(T, "_queue", record)
    monkeypatch.setattr(T.AdamW, "_tensor", lambda *a: None)
    return made


@pytest.mark.parametrize("state", ["f32", "f8"])
def test_adamw_follows_every_tensor_that_gets_other_storage(state, calls):
    """Parameters, copies and moments alike: what a call gets is where they are now, and never where they were."""
    params = [torch.zeros(300), torch.zeros(40)]
    opt = T.AdamW(params, lr=1e-3, state=state, copies=[torch.zeros(300, dtype=torch.bfloat16), None])
    grads = [torch.zeros(300), torch.zeros(40)]
    held = opt.states()

    def now():
        want = [dict(p=params[i], copy=opt.copies[i], **{k: t[i] for k, t in held.items()}) for i in range(2)]
        return [{k: None if t is None else t.data_ptr() for k, t in w.items()} for w in want]
    before = []                                          # what was there stays alive, so that no address is handed out twice
    for key, i in [(None, 0), ("p", 1), ("copy", 0), *((k, i) for k in held for i in (0, 1))]:
        if key is not None:
            t = params[i] if key == "p" else opt.copies[i] if key == "copy" else held[key][i]
            before.append(t.data)
            t.data = t.data.clone()
        opt.step(grads)
        if state == "f8":
            opt.read_moments()
        for made in calls:
            assert [{k: m[k] for k in w} for m, w in zip(made, now())] == now(), (key, i)
        calls.clear()


def test_adamw_refuses_a_tensor_that_comes_to_lie_on_another(calls):
    params = [torch.zeros(30), torch.zeros(30)]
    opt = T.AdamW(params, lr=1e-3)
    opt.step([torch.zeros(30)] * 2)
    params[1].data = opt.states()["v"][0].data
    for _ in range(2):
        with pytest.raises(ValueError):
            opt.step([torch.zeros(30)] * 2)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_choices_among_equal_logits_are_those_of_the_lowest_index(dtype):
    z = torch.tensor([[1.0, 3.0, 3.0, 0.0, 3.0], [2.0] * 5, [float("-inf")] * 5, [0.0, 1.0, -1.0, 1.0, 5.0]], dtype=dtype)
    got = T._choices(z, 3)
    assert got.dtype == torch.int32 and got.stride(1) == 1
    assert got.tolist() == [[1, 2, 4], [0, 1, 2], [0, 1, 2], [4, 1, 3]]
