"""Verification of drafted tokens in rows far longer than a vocabulary: what decides there is as exact as elsewhere, and takes time in proportion."""
import math
import time

import pytest
import torch

pytestmark = pytest.mark.gpu

BLOCK = 256


@pytest.fixture(scope="module")
def e3():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2505_18573_b200 import binding
    binding.lib()
    return binding


def test_sums_over_a_billion_entries(e3):
    """Every block holds one logit 0 and 255 of -x, so p(0) is known; uniforms within 1e-5 and 2e-5 of it.  Adding up 43,691 equal parts of such a row in
    fp32 is off by up to 2e-5, upwards or downwards by x."""
    V, k = 1 << 30, 1
    gaps = [s * g for g in (8e-6, 1.6e-5) for s in (1, -1)]
    for x in (4.6875, 4.65625):
        n = len(gaps)
        logits = torch.full((n * (k + 1), V), -x, device="cuda", dtype=torch.bfloat16)
        logits[:, ::BLOCK] = 0.0
        p = 1.0 / (V // BLOCK * (1.0 + 255.0 * math.exp(-x)))
        u = torch.full((n, k + V // BLOCK + 1), 0.5, device="cuda", dtype=torch.float64)
        u[:, 0] = torch.tensor([p * (1 + g) for g in gaps], dtype=torch.float64)
        u[:, k + 77] = 1 - 1e-12  # (the block that is drawn from)
        tok = torch.full((n, k), 5 * BLOCK, device="cuda", dtype=torch.int32)
        out, kept, logp, ent = e3.e3_verify_drafts(logits, torch.ones(n, device="cuda"), tok, u)
        assert kept.tolist() == [int(g < 0) for g in gaps]
        want = [math.log(p) if g < 0 else math.nan for g in gaps]
        for b in range(n):
            assert out[b, kept[b]].item() // BLOCK == 77
            if kept[b]:  # fp32 holds a logarithm of 20 to 2^-23 of it; 1e-5 for the sums, as in every row
                assert abs(logp[b, 0].item() - want[b]) <= 1e-5 + abs(want[b]) * 2.0 ** -23
        del logits
    torch.cuda.empty_cache()


def test_a_draft_like_the_target_in_a_long_row(e3):
    """Nothing is left of p - q, in any of 524,288 blocks: each is looked at a few times (0.5 s), not once for every other (half a minute)."""
    V, n, k = 1 << 27, 1, 1
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    logits = torch.randn((n * (k + 1), V), generator=g, device="cuda", dtype=torch.bfloat16)
    tok = torch.full((n, k), 1000, device="cuda", dtype=torch.int32)
    z = logits[0].double()
    logp = (z[1000] - z.logsumexp(0)).float().view(1, 1) + 1e-3  # q = 1.001 p
    u = torch.rand((n, k + V // BLOCK + 1), generator=g, device="cuda", dtype=torch.float64)
    u[:, 0] = 1 - 1e-9
    torch.cuda.synchronize()
    begin = time.perf_counter()
    out, kept, _, _ = e3.e3_verify_drafts(logits, torch.ones(n, device="cuda"), tok, u, draft_logits=logits[:1], draft_logp=logp)
    torch.cuda.synchronize()
    assert time.perf_counter() - begin < 4.0
    assert kept.item() == 0
    # nothing left: the draw is from p
    sums = torch.exp(z.view(-1, BLOCK) - z.max()).sum(1)
    score = sums.log() - (-u[0, 1:-1].log()).log()
    block = int(score.argmax())
    prefix = torch.exp(z.view(-1, BLOCK)[block] - z.max()).cumsum(0)
    assert out[0, 0].item() == block * BLOCK + int((prefix > u[0, -1] * prefix[-1]).int().argmax())
