"""The large tiles of the operators that train a layer's experts, which training runs on: whole numbers, which float holds whatever the order, and
the orthogonalising iteration in 64 bits.  Each test says which kernel it means and asks the profiler whether that one ran."""
import math
import re
import time

import pytest
import torch

from .test_gpu_expert_training import TYPES, U, bounds, i32, orthogonal

pytestmark = pytest.mark.gpu


def launched(call, *parts):
    """What call() returns, and the names of the device's kernels that it ran, with template arguments; a session that lacks one of these parts
    of names is repeated, since the profiler can miss what is close to its ends."""
    from torch.profiler import ProfilerActivity, profile
    for _ in range(4):
        torch.cuda.synchronize()
        with profile(activities=[ProfilerActivity.CUDA]) as prof:
            time.sleep(0.05)
            result = call()
            torch.cuda.synchronize()
            time.sleep(0.05)
        names = [e.name for e in prof.events()]
        if all(any(p in n for n in names) for p in parts):
            break
    return result, names


KINDS = ["SQUARE", "POLYNOMIAL", "APPLY", "RESULT"]


def muon_tiles(names):
    """{kind of product: tiles that it was done by}, and for how many stacks the launches were made."""
    tiles, stacks = {}, set()
    for n in names:
        m = re.search(r"muon_product_kernel<(\d+), \d+, \d+, \d+, [^0-9]*(\d), (\d+)>", n)
        if m:
            tiles.setdefault(KINDS[int(m[2])], set()).add(int(m[1]))
            stacks.add(int(m[3]))
    return tiles, stacks


# stacks of matrices; tiles of X X^T, of B, of B X, of the last product; how many stacks a launch's arguments hold
STACKS = [([(42, 521, 1003)], (256, 256, 256, 128), 1),
          ([(28, 520, 695)], (128, 128, 256, 128), 1),
          ([(20, 1003, 521), (11, 600, 1001), (11, 521, 1024)], (256, 256, 256, 128), 4),
          ([(9, 521, 1003), (9, 1003, 521), (8, 530, 1000), (8, 999, 700), (8, 768, 1010)], (256, 256, 256, 128), 24)]


@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("shapes,tiles,held", STACKS, ids=str)
def test_muon_by_large_tiles(shapes, tiles, held, grad):
    """One step of one to five stacks, wide and upright, of sizes that are no multiples of a tile: the first matrix of each against the iteration in
    64 bits, all of them against orthogonalise of one at a time, which takes other tiles and has the same bits before its rounding."""
    from paper_2603_19289_amd import training as T
    g = torch.Generator("cuda").manual_seed(len(shapes) * 100 + shapes[0][0])
    p = [torch.randn(s, generator=g, device="cuda") * 0.1 for s in shapes]
    grads = [torch.randn(s, generator=g, device="cuda").to(TYPES[grad]) for s in shapes]
    before = [t.double() for t in p]
    lr, decay, rms = 0.1, 0.3, 0.2

    def step():
        for t, b in zip(p, before):
            t.copy_(b)
        T.Muon(p, lr=lr, momentum=0.0, nesterov=False, weight_decay=decay, update_rms=rms, copies=copies).step(grads)
    copies = [torch.zeros(s, device="cuda", dtype=torch.bfloat16) for s in shapes]
    _, names = launched(step, *(f"MuonProduct){i}," for i in range(4)))
    assert muon_tiles(names) == ({k: {t} for k, t in zip(KINDS, tiles)}, {held}), sorted(set(names))
    for s, t, b, v, c in zip(shapes, p, before, grads, copies):
        rate = lr * rms * math.sqrt(max(s[1:]))
        assert torch.equal(c, t.to(torch.bfloat16))
        o, err = orthogonal(v[0].cpu())
        want = b[0].cpu() * (1 - lr * decay) - rate * o
        off = (t[0].cpu().double() - want).norm().item()
        assert off <= rate * err + 4 * U * (b[0].norm().item() + rate * o.norm().item()), (s, off, rate * err)
        for i in range(s[0]):
            o = T.orthogonalise(v[i]).double()
            step_of = 2.0 ** -8 * o.abs() / (1 - 2.0 ** -8)               # the rounding to bfloat16
            bound = rate * step_of + 4 * U * (b[i].abs() + rate * o.abs())
            assert ((t[i].double() - (b[i] * (1 - lr * decay) - rate * o)).abs() <= bound).all(), (s, i)
