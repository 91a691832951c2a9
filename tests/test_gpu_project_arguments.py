"""The projection's status word, and its scales at the ends of the range of fp32."""
import pytest
import torch

from test_gpu_project import check, operands, values

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def e3():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2505_18573_b200 import binding
    binding.lib()
    return binding


@pytest.mark.parametrize("rows", [5, 100, 300])
def test_status_words_of_a_larger_tensor(e3, rows):
    """As for the row calls: an int32 tensor whose first entry is the word."""
    ops = operands(1, rows, 300, 200)
    status = torch.tensor([0, 7, 9], device="cuda", dtype=torch.int32)
    want = e3.e3_project_vocab(*ops)
    assert torch.equal(e3.e3_project_vocab(*ops, status=status), want) and status.tolist() == [0, 7, 9]
    for bad in (status.long(), status[:0]):
        with pytest.raises(ValueError):
            e3.e3_project_vocab(*ops, status=bad)


@pytest.mark.parametrize("rows", [5, 100, 300])
def test_scales_whose_product_fp32_holds(e3, rows):
    """Far from 1 each, near 1 together."""
    for up in (100.0, -100.0):
        x, sx, w, sw = operands(2, rows, 300, 500)
        check(e3, (x, sx * 2.0 ** up, w, sw * 2.0 ** -up), torch.float32)


@pytest.mark.parametrize("rows", [5, 100, 300])
def test_scales_whose_product_fp32_does_not_hold(e3, rows):
    """The two scales of a block are multiplied in fp32 first: from 2^128 on the logits of the block are not finite, below 2^-149 it adds nothing."""
    x, sx, w, sw = operands(3, rows, 300, 500)
    sx[2, 1], sw[1, 1] = 2.0 ** 120, 2.0 ** 100
    sw[0, 1], sw[2, 1] = 2.0 ** -120, 2.0 ** -119
    got = e3.e3_project_vocab(x, sx, w, sw, dtype=torch.float32)
    bad = torch.zeros((rows, 300), dtype=torch.bool, device="cuda")
    bad[2, 128:256] = True
    assert torch.equal(~got.isfinite(), bad)
    sx, sw = torch.full_like(sx, 2.0 ** -80), torch.full_like(sw, 2.0 ** -80)
    sx[:, 3] = 1.0
    a, b = values(x, torch.where(torch.arange(4, device="cuda") == 3, sx, 0.0), 1), values(w, sw, 128)
    # as in `check`: a block's additions, each within 2^-23 of the sum of absolute values, two scales, the sum over four blocks, the output
    bound = (a.abs() @ b.abs().t()) * (128 * 2.0 ** -23 + 8 * 2.0 ** -24)
    assert bool(((e3.e3_project_vocab(x, sx, w, sw, dtype=torch.float32).double() - a @ b.t()).abs() <= bound).all())
