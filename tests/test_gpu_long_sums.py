"""Long sums of float products in every kernel that makes them.  All terms are 1 + 2^-14: in one running float sum the 2^-14 is lost from 4096 on
(four terms together are then half a step or less: a tie, which goes to the even value, that they start from), which leaves three quarters of it out of
16384 terms and half of it out of 8192, 4.5e-5 and 3.0e-5 of the result."""
import pytest
import torch

from .test_gpu_expert_training import U, i32
from .test_gpu_expert_training_large import launched

pytestmark = pytest.mark.gpu

LONG = 65536


@pytest.mark.parametrize("transpose,rows,short,kernel,run,joined", [
    (False, 3, 40, "grouped_few_kernel<float>", 256, 64 + 4), (True, 3, 40, "grouped_few_transposed_kernel", 64, 128 + 8),
    (False, 300, 40, "grouped_kernel<moe_spec::F32", 256, 256), (True, 300, 40, "grouped_kernel<moe_spec::F32", 256, 256),
    (False, 300, 39, "grouped_f32_kernel", 256, 256), (True, 300, 39, "grouped_f32_kernel", 256, 256)])
def test_long_sums_of_products(transpose, rows, short, kernel, run, joined):
    """A cut inside a matrix instruction counts twice a rounding: 2 u for each product of a run, u for each run that is added up."""
    from paper_2603_19289_amd import training as T
    long = LONG if short % 4 == 0 or transpose else LONG - 1          # rows of the operands that are no multiples of 16 bytes
    x = torch.ones(rows, long, device="cuda")
    w = torch.full((1, long, short) if transpose else (1, short, long), 1 + 2.0 ** -14, device="cuda")
    y, names = launched(lambda: T.grouped_product(x, w, i32([rows]), transpose=transpose), kernel)
    assert any(kernel in v for v in names), sorted(set(names))
    want = long * (1 + 2.0 ** -14)
    assert ((y.double() - want).abs() <= (2 * run + joined + 8) * U * want).all(), ((y.double() - want).abs().max() / want).item()


@pytest.mark.parametrize("n,k,kernel,parts", [(72, 136, "weight_grad_kernel<moe_spec::F32", 64), (2048, 2052, "weight_grad_kernel<moe_spec::F32", 1), (71, 135, "weight_grad_f32_kernel", 64)])
def test_long_sums_of_weight_gradients(n, k, kernel, parts):
    from paper_2603_19289_amd import training as T
    dy, x = torch.ones(LONG, n, device="cuda"), torch.full((LONG, k), 1 + 2.0 ** -14, device="cuda")
    dw, names = launched(lambda: T.grouped_weight_grad(dy, x, i32([LONG])), kernel)
    assert any(kernel in v for v in names), sorted(set(names))
    want = LONG * (1 + 2.0 ** -14)
    assert ((dw.double() - want).abs() <= (2 * 256 + 256 + parts + 8) * U * want).all(), ((dw.double() - want).abs().max() / want).item()
