"""Embedding, 8-bit projection, sampling and verification together, as a rollout with drafted tokens and the training step behind it use them."""
import math
import types

import numpy as np
import pytest
import torch

from _compare import assert_close
from test_gpu_project import values
from test_gpu_verify import BLOCK, reference

pytestmark = pytest.mark.gpu

N, K, V, D, DRAFT_D = 7, 3, 1500, 200, 72
SCALE = 3.0


@pytest.fixture(scope="module")
def e3():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2505_18573_b200 import binding
    binding.lib()
    return binding


class Model:
    """Logits of a token from its own embedding; one table at both ends, in 8 bits at the second."""

    def __init__(self, e3, table, dtype, scale=SCALE):
        self.e3, self.table, self.dtype, self.scale = e3, table, dtype, scale
        self.w, self.sw = e3.e3_quantize(table, block_rows=128)

    def __call__(self, tok):
        self.hidden = self.e3.e3_embed_tokens(self.table, tok.reshape(-1), self.scale)
        self.x, self.sx = self.e3.e3_quantize(self.hidden)
        self.logits = self.e3.e3_project_vocab(self.x, self.sx, self.w, self.sw, dtype=self.dtype)
        return self.logits

    def check(self, tok):
        """The last call in 64 bits, through the values that the 8 bits stand for."""
        assert torch.equal(self.hidden, (self.table.float()[tok.reshape(-1).long()] * self.scale).to(self.table.dtype))
        a, b = values(self.x, self.sx, 1), values(self.w, self.sw, 128)
        # a block's largest entry becomes 224 to 448, and 4 bits of it are kept: half a step, 2^-4 of the value, or of the smallest normal 2^-6,
        # which is at most 2^-6 / 224 of the block's largest
        for stands, real in ((a, self.hidden.double()), (b, self.table.double())):
            assert bool(((stands - real).abs() <= real.abs() * 2.0 ** -4 + real.abs().max() * 2.0 ** -10 / 224).all())
        want, size = a @ b.t(), a.abs() @ b.abs().t()
        sums = size * (128 * 2.0 ** -23 + (self.sx.shape[1] + 3) * 2.0 ** -24)  # as for the projection alone
        assert bool(((self.logits.double() - want).abs() <= sums + (want.abs() + sums) * torch.finfo(self.dtype).eps / 2).all())


def tables(dtype):
    g = torch.Generator(device="cuda")
    g.manual_seed(7)
    table = torch.randn((V, D), generator=g, device="cuda") * 0.35
    draft = torch.randn((V, DRAFT_D), generator=g, device="cuda") * 0.35
    draft[:, :DRAFT_D // 2] = table[:, :DRAFT_D // 2] * 1.5  # the drafts agree with the target in part
    return table.to(dtype), draft.to(dtype), g


def step(e3, target, drafter, cur, temps, uniforms, counter):
    """K tokens drafted one after the other, then one call over all of them: the drafter's inputs and the outputs of the verification."""
    toks, logits, logps = [cur], [], []
    for j in range(K):
        logits.append(drafter(toks[-1]))
        tok, logp, _ = e3.e3_sample(logits[-1], temps, 11, counter + j)
        toks.append(tok)
        logps.append(logp)
    draft_tok, draft_logp = torch.stack(toks[1:], 1), torch.stack(logps, 1)
    draft_logits = torch.stack(logits, 1).reshape(N * K, V)
    seen = torch.stack(toks, 1)
    out = e3.e3_verify_drafts(target(seen), temps, draft_tok, uniforms, draft_logits=draft_logits, draft_logp=draft_logp)
    return seen, draft_tok, draft_logits, draft_logp, out


@pytest.mark.parametrize("scale", [SCALE, 0.25])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_rollout_with_drafts(e3, dtype, scale):
    table, draft, g = tables(dtype)
    target, drafter = Model(e3, table, dtype, scale), Model(e3, draft, dtype, scale)
    temps = torch.linspace(0.6, 1.4, N, device="cuda")
    cur = torch.randint(0, V, (N,), generator=g, device="cuda", dtype=torch.int32)
    total = 0
    for at in range(6):
        uniforms = torch.rand((N, K + -(-V // BLOCK) + 1), generator=g, device="cuda", dtype=torch.float64)
        seen, draft_tok, draft_logits, draft_logp, (tok, kept, logp, ent) = step(e3, target, drafter, cur, temps, uniforms, at * K)
        target.check(seen)
        drafter.check(seen[:, K - 1])
        want = reference(types.SimpleNamespace(n=N, k=K, V=V, logits=target.logits, temps=temps, draft_tok=draft_tok, uniforms=uniforms,
                                               draft_len=None, draft_logits=draft_logits, draft_temps=None, draft_logp=draft_logp))
        assert np.array_equal(kept.cpu().numpy(), want[1]) and np.array_equal(tok.cpu().numpy(), want[0])
        assert_close("logp", logp.cpu().numpy(), want[2], 1e-5)
        assert_close("ent", ent.cpu().numpy(), want[3], 1e-5)
        # the training forward reads the same logits; both are within 1e-5
        rows = (tok >= 0).reshape(-1)
        again = e3.e3_token_logp_entropy(target.logits, tok.clamp_min(0).reshape(-1), mask=rows.to(torch.uint8), temps=temps.repeat_interleave(K + 1))
        assert_close("logp", again[0][rows].cpu().numpy(), logp.reshape(-1)[rows].cpu().numpy(), 2e-5)
        assert_close("ent", again[1][rows].cpu().numpy(), ent.reshape(-1)[rows].cpu().numpy(), 2e-5)
        total += int(kept.sum())
        cur = tok.gather(1, kept[:, None].long()).squeeze(1).contiguous()
        assert bool((cur >= 0).all())
    # a token's logit of itself is scale * 200 * 0.35^2, the others' spread scale * 0.35^2 * sqrt(200): at 3.0 73 against 5, so that both models repeat it and
    # every draft is kept; at 0.25 6.1 against 0.4, a probability of about 0.2, and the drafter's half as much in its exponent, so that some are not
    assert total == 6 * N * K if scale == SCALE else 0 < total < 6 * N * K


def test_a_captured_step_replays_on_new_tokens(e3):
    table, draft, g = tables(torch.bfloat16)
    target, drafter = Model(e3, table, torch.bfloat16), Model(e3, draft, torch.bfloat16)
    temps = torch.linspace(0.6, 1.4, N, device="cuda")
    cur = torch.randint(0, V, (N,), generator=g, device="cuda", dtype=torch.int32)
    uniforms = torch.rand((N, K + -(-V // BLOCK) + 1), generator=g, device="cuda", dtype=torch.float64)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(e3, target, drafter, cur, temps, uniforms, 5)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = step(e3, target, drafter, cur, temps, uniforms, 5)
    torch.cuda.current_stream().wait_stream(side)
    for _ in range(3):
        cur.copy_(torch.randint(0, V, (N,), generator=g, device="cuda", dtype=torch.int32))
        uniforms.copy_(torch.rand(uniforms.shape, generator=g, device="cuda", dtype=torch.float64))
        graph.replay()
        got = [x.clone() for x in out[4]]
        want = step(e3, target, drafter, cur, temps, uniforms, 5)
        assert all(torch.equal(a, b) for a, b in zip(got, want[4])) and torch.equal(out[0], want[0])


def objective(table, stands, off, b, seen, tok, mask, temps, logp_old, adv, clip):
    """The objective of the table's rows alone (`stands`: the hidden states' values in 8 bits, `off`: how far the delivered logits are from their products, both
    passed through in the gradient), in 64 bits."""
    hidden = SCALE * table[seen.reshape(-1).long()]
    x = hidden + (stands - hidden).detach()
    z = x @ b.t()
    z = (z + off) / temps.double()[:, None]
    logp = z.log_softmax(-1).gather(1, tok.reshape(-1, 1).long()).reshape(seen.shape)
    ratio = torch.exp(logp - logp_old.double())
    a = adv.double()[:, None]
    terms = torch.minimum(ratio * a, ratio.clamp(1 - clip, 1 + clip) * a) * mask
    return (terms.sum(1) / mask.sum(1).clamp_min(1)).mean()


def test_the_gradient_of_a_training_step(e3):
    """Objective -> logits -> hidden states (products of the caller's, here in 64 bits) -> table, against the formula and differences."""
    table, _, g = tables(torch.float32)
    target = Model(e3, table, torch.float32)
    T = 9
    seen = torch.randint(0, 40, (N, T), generator=g, device="cuda", dtype=torch.int32)  # tokens that come more than once
    mask = (torch.arange(T, device="cuda")[None] < torch.randint(1, T + 1, (N, 1), generator=g, device="cuda")).to(torch.uint8)
    seen = torch.where(mask.bool(), seen, torch.full_like(seen, -1))  # padding
    tok = torch.randint(0, V, (N, T), generator=g, device="cuda", dtype=torch.int32)
    temps = torch.linspace(0.6, 1.4, N, device="cuda").repeat_interleave(T)
    adv = torch.linspace(-1.5, 1.5, N, device="cuda")
    logits = target(seen)
    logp, ent = e3.e3_token_logp_entropy(logits, tok.reshape(-1), mask=mask.reshape(-1), temps=temps)[:2]
    logp_old = (logp.reshape(N, T) + 0.02 * torch.randn((N, T), generator=g, device="cuda")) * mask
    offsets = torch.tensor([0, N], dtype=torch.int64, device="cuda")
    (J, g_logp) = e3.e3_grpo_objective(logp.reshape(N, T), logp_old, adv, offsets, mask=mask)
    dlogits = e3.e3_token_logp_entropy_backward(logits, tok.reshape(-1), logp, ent, g_logp=g_logp.reshape(-1), mask=mask.reshape(-1), temps=temps)
    b = values(target.w, target.sw, 128)
    dhidden = (dlogits.double() @ b).float()
    got = e3.e3_embed_tokens_backward(dhidden, seen.reshape(-1), V, SCALE)

    stands = values(target.x, target.sx, 1)
    leaf = table.double().requires_grad_()
    live = seen.clamp_min(0)
    off = logits.double() - stands @ b.t()
    args = (stands, off, b, live, tok, mask.double(), temps, logp_old, adv, 0.2)
    value = objective(leaf, *args)
    value.backward()
    # padded positions are masked, so the row that stands in for -1 gets nothing from them
    # logits / tau and logp are below 2^8, so that four fp32 roundings of them and 1e-5 for the sum are 4e-5 of a weight (as an exponent's error) and of the
    # objective's ratio; then four fp32 roundings on the way
    p = (logits.double() / temps.double()[:, None]).softmax(-1)
    hot = torch.zeros_like(p).scatter_(1, tok.reshape(-1, 1).long(), 1.0)
    weight = (g_logp.double().abs().reshape(-1) / temps.double())[:, None]
    err = (weight * (4e-5 * p + (4e-5 + 4 * 2.0 ** -24) * (hot - p).abs())) @ b.abs()
    size = dhidden.double().abs()
    bound = torch.zeros((V, D), dtype=torch.float64, device="cuda")
    live_rows = mask.reshape(-1).bool()
    count = live_rows.sum()
    bound.index_add_(0, live.reshape(-1)[live_rows].long(), SCALE * (err + (count + 3) * 2.0 ** -24 * size)[live_rows])
    diff = (got.double() - leaf.grad).abs()
    assert bool((diff <= bound * 1.01).all()), float((diff / bound.clamp_min(1e-300)).max())
    assert bool((got[seen[adv != 0][mask[adv != 0].bool()].unique().long()] != 0).any(1).all())
    # the same along one direction, by central differences: the objective's third derivative times h^2 is far below the tolerance
    way = torch.zeros_like(leaf)
    way[:40] = torch.randn((40, D), generator=g, device="cuda", dtype=torch.float64)
    h = 1e-5

    def moved(s):
        at = table.double() + s * way
        return objective(at, stands + SCALE * s * way[live.reshape(-1).long()], *args[1:])

    slope = float(moved(h) - moved(-h)) / (2 * h)
    assert math.isclose(slope, float((got.double() * way).sum()), rel_tol=1e-4, abs_tol=float((bound * way.abs()).sum()) + 1e-7)
