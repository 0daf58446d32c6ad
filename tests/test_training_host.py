"""What training.py does on the host, on a machine without a GPU: calls into the library are recorded instead of made, and the checks that
tensors lie on a GPU are left out."""
import os
import subprocess

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


DEALING = r"""
#include <cstdio>
#include <vector>
#include "train_rules.h"
using namespace moe_spec;
int main() {
  int bad = 0;
  const int64_t most = MOE_SPEC_ADAMW_MAX_ELEMENTS;
  const int64_t lists[][4] = {{0, 1, 2048, 2049}, {most, most, 1, most}, {most / 2, most / 2, 4096, most}, {1, most, 1, 0},
                              {most - 2048, 2048, 1, 5}, {most - 2048, 2049, 1, 5}, {0, 0, 0, 0}, {5, 0, 0, 7}};
  for (auto &sizes : lists) for (int n : {0, 1, 4, 39, 40, 41, 80, 81, 300}) {
    std::vector<moe_spec_adamw_tensor> t(n);
    for (int i = 0; i < n; ++i) t[i].n = sizes[i % 4];
    int next = 0, slots = 0, launches = 0;
    int64_t blocks = 0;
    bool ok = true;
    in_launches(t.data(), n, [&](int slot, int i, uint32_t first) {
      while (next < i && t[next].n == 0) ++next;              // what lies between has no elements
      ok = ok && slot == slots++ && i == next++ && t[i].n > 0 && int64_t(first) == blocks;
      blocks += (t[i].n + kAdamChunk - 1) / kAdamChunk;
    }, [&](int count, unsigned grid) {
      ok = ok && count == slots && count >= 1 && count <= kPerLaunch && int64_t(grid) == blocks && uint64_t(grid) * kAdamBlock < (uint64_t(1) << 32);
      slots = 0;
      blocks = 0;
      ++launches;
      return 0;
    });
    while (next < n && t[next].n == 0) ++next;
    if ((!ok || next != n || slots) && ++bad <= 20) std::printf("n %d, first %lld: %d launches, next %d\n", n, (long long)sizes[0], launches, next);
    int calls = 0;
    const int e = in_launches(t.data(), n, [](int, int, uint32_t) {}, [&](int, unsigned) { return ++calls == 2 ? 7 : 0; });
    if ((launches >= 2 ? e != 7 || calls != 2 : e != 0 || calls != launches) && ++bad <= 20) std::printf("n %d: status %d after %d calls\n", n, e, calls);
  }
  return bad ? 1 : 0;
}
"""


def test_adamw_tensors_are_dealt_to_launches_that_fit(tmp_path):
    """Every tensor that has elements is in exactly one launch, in order, its workgroups behind those of the tensors before it; a
    launch has at most an argument block's tensors and fewer than 2^32 threads; one that fails ends the call."""
    src, exe = tmp_path / "deal.cpp", tmp_path / "deal"
    src.write_text(DEALING)
    csrc = os.path.join(os.path.dirname(M.__file__), "csrc")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", csrc, str(src), "-o", str(exe)], check=True)
    done = subprocess.run([str(exe)], capture_output=True, text=True, timeout=120)
    assert done.returncode == 0, done.stdout[-2000:]


def test_moments_are_read_into_the_tensors_that_are_named(monkeypatch):
    """One list of outputs, the other or both: the addresses that the library gets, and a list of the wrong length."""
    got = []
    monkeypatch.setattr(T, "_queue", lambda dev, call, desc, n, dtype, m, v: got.append([None if a is None else list(a) for a in (m, v)]))
    monkeypatch.setattr(T.AdamW, "_tensor", lambda *a: None)
    sizes = (300, 40, 7)
    opt = T.AdamW([torch.zeros(n) for n in sizes], lr=1e-3, state="f8")
    m, v = ([torch.zeros(n, dtype=torch.bfloat16) for n in sizes] for _ in range(2))
    at = lambda out: [t.data_ptr() for t in out]  # noqa: E731
    assert opt.read_moments(m, v) == (m, v) and opt.read_moments(m) == (m, None) and opt.read_moments(v_out=tuple(v)) == (None, tuple(v))
    new = opt.read_moments()
    assert got == [[at(m), at(v)], [at(m), None], [None, at(v)], [at(new[0]), at(new[1])]]
    for bad in ((m[:2], v + v[:1]), (m[:2], None), (None, [])):
        with pytest.raises(ValueError):
            opt.read_moments(*bad)
