"""Verification of drafted tokens where its contract ends: uniforms of exactly 0, weights that fp32 cannot hold."""
import math

import numpy as np
import pytest
import torch

from test_gpu_verify import BLOCK, INF, Batch, host, reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def e3():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2505_18573_b200 import binding
    binding.lib()
    return binding


def same(got, want):
    """Equal tokens and counts; logarithms and entropies of calls that may have taken the normaliser in 32 and in 64 bits, either within 1e-5 of the
    definition (as `check` has them) and so within 2e-5 of each other."""
    return (torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and
            all(torch.allclose(x, y, rtol=0.0, atol=2e-5, equal_nan=True) for x, y in zip(got[2:], want[2:])))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("model", [True, False])
@pytest.mark.parametrize("V", [1, 200, 256])
def test_one_block_and_its_uniform_0(e3, dtype, model, V):
    """A single block is drawn from whatever its uniform is."""
    s = Batch(V, 20, 2, V, dtype, model)
    s.uniforms[:, 2] = 0.5
    want = s.check(e3)
    s.uniforms[:, 2] = 0.0
    assert same(s.call(e3), want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_one_block_left_by_the_mask_and_its_uniform_0(e3, dtype):
    for V, alive in ((3000, 4), (3000, 11), (540000, 2100)):
        s = Batch(V, 6, 1, V, dtype, model=False)
        row = torch.full_like(s.logits, -INF)
        row[:, alive * BLOCK:(alive + 1) * BLOCK] = s.logits[:, alive * BLOCK:(alive + 1) * BLOCK]
        s.logits = row
        s.draft_tok.fill_(0)  # (masked: refused)
        want = s.check(e3)
        s.uniforms[:, 1 + alive] = 0.0
        assert same(s.call(e3), want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("first", [0, 2])
def test_uniforms_of_0_alone_give_the_first_block_that_has_weight(e3, dtype, first):
    s = Batch(3, 8, 0, 2000, dtype, model=False)
    s.logits[:, :first * BLOCK] = -INF
    s.uniforms[:, :-1] = 1e-300
    s.uniforms[:, first] = 1 - 1e-12
    want = s.check(e3)
    assert bool((want[0] // BLOCK == first).all())
    s.uniforms[:, :-1] = 0.0
    assert same(s.call(e3), want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("model", [True, False])
def test_what_is_left_of_a_refused_draft_lies_in_a_block_with_the_uniform_0(e3, dtype, model):
    """The draft has one block, the target that and another: the other is drawn from, and not the refused token again."""
    n, V = 10, 1500
    s = Batch(4, n, 1, V, dtype, model)
    z = torch.full((n, 2, V), -INF, device="cuda")
    for b in range(n):
        z[b, :, 2 * BLOCK + 7], z[b, :, 4 * BLOCK:4 * BLOCK + 40 + b] = 2.0, -1.0
    s.logits = z.view(2 * n, V).to(dtype)
    s.draft_tok.fill_(2 * BLOCK + 7)
    s.temps.fill_(1.0)
    if model:
        y = torch.full((n, V), -INF, device="cuda")
        y[:, 2 * BLOCK + 7] = 1.0
        s.draft_logits, s.draft_logp, s.draft_temps = y.to(dtype), torch.zeros((n, 1), device="cuda"), s.temps
    s.uniforms[:, 0] = 0.999
    want = s.check(e3)
    assert bool((want[0][:, 0] // BLOCK == 4).all())
    s.uniforms[:, 1 + 4] = 0.0
    assert same(s.call(e3), want)
    s.uniforms[:, 1:-1] = 0.0
    assert same(s.call(e3), want)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_what_is_left_is_less_than_fp32_holds(e3, dtype):
    """All of the target's mass at the draft, whose q is as large; what is left are the other entries' exp(-100)."""
    n, V = 16, 9 * BLOCK - 30
    s = Batch(5, n, 1, V, dtype)
    z = torch.full((n, 2, V), -100.0, device="cuda")
    z[:, :, BLOCK:2 * BLOCK], z[:, :, 8 * BLOCK:] = -INF, -INF
    z[:, :, BLOCK + 3] = 0.0
    s.logits = z.view(2 * n, V).to(dtype)
    y = torch.full((n, V), -INF, device="cuda")
    y[:, BLOCK + 3] = 0.0
    s.draft_logits, s.draft_tok, s.temps = y.to(dtype), torch.full_like(s.draft_tok, BLOCK + 3), torch.ones_like(s.temps)
    s.draft_temps, s.draft_logp = s.temps, torch.full((n, 1), 1e-3, device="cuda")  # (q a thousandth above p)
    s.uniforms[:, 0] = 1 - 1e-9
    tok, kept, _, _ = s.call(e3)
    want = reference(s)
    assert not kept.any() and np.array_equal(tok.cpu().numpy(), want[0])
    assert not bool((tok[:, 0] == BLOCK + 3).any())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("alone", [-83.0, -60.0, -90.0])
def test_weights_that_fp32_holds_beside_weights_that_it_does_not(e3, dtype, alone):
    """Nothing left at the draft; one entry of exp(alone) in a block, 256 of exp(-88) in another: fp32 holds exp(-83), but neither exp(-88) nor its sum's terms."""
    n, V = 12, 6 * BLOCK
    s = Batch(8, n, 1, V, dtype)
    z = torch.full((n, 2, V), -INF, device="cuda")
    z[:, :, 5 * BLOCK + 3], z[:, :, BLOCK + 9], z[:, :, 4 * BLOCK:5 * BLOCK] = 0.0, alone, -88.0  # (0 and -88 under one reference)
    s.logits = z.view(2 * n, V).to(dtype)
    y = torch.full((n, V), -INF, device="cuda")
    y[:, 5 * BLOCK + 3] = 0.0
    s.draft_logits, s.draft_tok, s.temps = y.to(dtype), torch.full_like(s.draft_tok, 5 * BLOCK + 3), torch.ones_like(s.temps)
    s.draft_temps, s.draft_logp = s.temps, torch.full((n, 1), 1e-3, device="cuda")
    s.uniforms[:, 0], s.uniforms[:, 2], s.uniforms[:, 5] = 1 - 1e-9, 0.5, 0.5
    tok, kept, _, _ = s.call(e3)
    want = reference(s)
    assert not kept.any() and np.array_equal(tok.cpu().numpy(), want[0])
    assert bool((tok[:, 0] // BLOCK == (1 if alone == -60.0 else 4)).all())


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_greedy_sequences_look_at_no_uniforms_of_the_draw(e3, dtype):
    """At tau = 0 the token behind the kept drafts is the arg-max: of the uniforms only u_j has to lie in [0, 1)."""
    s = Batch(6, 12, 2, 900, dtype, greedy=1.0)
    want = s.check(e3)
    s.uniforms[:, 2:] = torch.tensor([math.nan, 1.0, -1.0, INF, 2.0], dtype=torch.float64, device="cuda")[:s.uniforms.shape[1] - 2]
    assert same(s.call(e3), want)
    s.uniforms[:, 0] = 1.0
    tok, kept, logp, ent = s.call(e3)
    assert bool((tok == -1).all()) and not kept.any() and bool(logp[:, 0].isnan().all()) and bool(ent[:, 0].isnan().all())
    assert host(tok).shape == (12, 3)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_log_probabilities_hang_on_the_row_alone(e3, dtype):
    """However near the draw's other candidates come: the same bits whether fp32 settles it or the row's normaliser is taken in fp64 for it."""
    s = Batch(7, 60, 1, 256, dtype)
    s.uniforms[:, 1] = 0.5
    want = s.call(e3)
    s.uniforms[:, 1] = 0.0  # (one block, whose score fp32 cannot tell from others')
    assert all(torch.equal(x, y) for x, y in zip(s.call(e3), want))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("error", [1e-5, 1e-3, 0.05])
def test_a_draft_almost_like_the_target(e3, dtype, error):
    """So little is left of p - q that most blocks' scores of p reach the best score of that, more than are taken in their order."""
    s = Batch(9, 4, 1, 400_000, dtype, error=error, sharp=0.2)
    s.draft_logp = s.draft_logp + 1e-4
    s.uniforms[:, 0] = 1 - 1e-9
    s.check(e3)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("tau", [1e-40, 1e-45, 4e-39, 1e-37])
def test_drafts_at_temperatures_next_to_0(e3, dtype, tau):
    """The draft's logits tie at three places, of a third each, however small its temperature: log2(e) / tau is beyond fp32 below 4.3e-39."""
    n, V = 32, 5 * BLOCK
    s = Batch(10, n, 1, V, dtype)
    places = [5, 3 * BLOCK + 1, 4 * BLOCK]
    z = torch.zeros((n, 2, V), device="cuda")
    z[:, :, places[0]], z[:, :, places[1]], z[:, :, places[2]] = 6.5, 8.25, 7.25
    s.logits = z.view(2 * n, V).to(dtype)
    y = torch.full((n, V), -3.0, device="cuda")
    y[:, places] = 1.5
    s.draft_logits, s.draft_tok, s.temps = y.to(dtype), torch.full_like(s.draft_tok, places[0]), torch.ones_like(s.temps)
    s.draft_temps, s.draft_logp = torch.full((n,), tau, device="cuda"), torch.full((n, 1), -math.log(3.0), device="cuda")
    s.uniforms[:, 0] = 0.9
    tok, kept, _, _ = s.check(e3)
    assert not kept.any() and 0 < int((tok[:, 0] == places[1]).sum()) < n
