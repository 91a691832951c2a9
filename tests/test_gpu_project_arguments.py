"""The projection's status word."""
import pytest
import torch

from test_gpu_project import operands

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
