"""Gradient of tokens with long runs, in whole numbers whose sums fp32 holds: equal, so that no segment of a run can be lost or taken twice."""
import pytest
import torch

from test_gpu_embed import generator

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def e3():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2505_18573_b200 import binding
    binding.lib()
    return binding


def check(e3, tok, V, D, seed, dtype):
    n = tok.numel()
    g = torch.randint(-3, 4, (n, D), generator=generator(seed), device="cuda").to(dtype)
    live = (tok >= 0) & (tok < V)
    want = torch.zeros((V, D), device="cuda", dtype=torch.float64).index_add_(0, tok[live].long(), g[live].double())
    assert float(want.abs().max()) < 2 ** 24  # (and so is every partial sum: at most 3 n)
    got = e3.e3_embed_tokens_backward(g, tok, V, dtype=torch.float32)
    assert torch.equal(got.double(), want)
    added = torch.randint(-1000, 1000, (V, D), generator=generator(seed + 1), device="cuda").float()
    assert torch.equal(e3.e3_embed_tokens_backward(g, tok, V, out=added.clone(), accumulate=True).double(), added.double() + want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("D", [3, 40])
@pytest.mark.parametrize("n", [31, 32, 33, 64, 129, 4096, 4097, 32767, 32768, 40000, 131072, 500001])
def test_one_token_alone(e3, n, D, dtype):
    check(e3, torch.full((n,), 3, device="cuda", dtype=torch.int32), 5, D, n, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [1000, 4096, 5000, 60000, 300000])
def test_runs_of_every_length(e3, n, dtype):
    """Tokens in order of frequency, as vocabularies number them: runs of half of all tokens down to one, neighbours in the table."""
    g = generator(n)
    tok = torch.exp(torch.rand(n, generator=g, device="cuda") * 9.0).int() - 1
    tok = torch.where(torch.rand(n, generator=g, device="cuda") < 0.02, -1, tok).int()
    check(e3, tok, 9000, 24, n, dtype)
    check(e3, torch.sort(tok).values, 9000, 24, n, dtype)
