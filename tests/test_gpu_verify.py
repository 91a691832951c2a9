"""Verification of drafted tokens against the definition in 64 bits, one sequence and one position after the other."""
import math

import numpy as np
import pytest
import torch

from _compare import assert_close

pytestmark = pytest.mark.gpu

BLOCK = 256
INF = math.inf


@pytest.fixture(scope="module")
def e3():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2505_18573_b200 import binding
    binding.lib()
    return binding


class Batch:
    """Inputs of a call, on the GPU; `arguments` as the binding takes them."""

    def __init__(self, seed, n, k, V, dtype=torch.float32, model=True, ragged=False, greedy=0.0, error=0.7, sharp=3.0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.n, self.k, self.V = n, k, V
        rand = lambda *s, **a: torch.rand(s, generator=g, device="cuda", **a)  # noqa: E731
        z = sharp * torch.randn((n * (k + 1), V), generator=g, device="cuda")
        self.logits = z.to(dtype)
        tau = rand(n) * 0.8 + 0.6
        self.temps = torch.where(rand(n) < greedy, torch.zeros_like(tau), tau)
        self.draft_len = torch.randint(0, k + 1, (n,), generator=g, device="cuda", dtype=torch.int32) if ragged else None
        self.draft_logits = self.draft_temps = self.draft_logp = None
        y = z.view(n, k + 1, V)[:, :k] + error * torch.randn((n, k, V), generator=g, device="cuda")
        if model:
            self.draft_logits, self.draft_temps = y.reshape(n * k, V).to(dtype), tau
            x = self.draft_logits.view(n, k, V).float() / tau[:, None, None]
            tok = (x - torch.log(-torch.log(rand(n, k, V).clamp_min(1e-20)))).argmax(-1) if k else torch.zeros((n, 0), device="cuda")
            self.draft_logp = x.gather(-1, tok[..., None].long()).squeeze(-1) - x.logsumexp(-1) if k else torch.zeros((n, 0), device="cuda")
        else:
            tok = torch.where(rand(n, k) < 0.7, z.view(n, k + 1, V)[:, :k].argmax(-1), torch.randint(0, V, (n, k), generator=g, device="cuda"))
        self.draft_tok = tok.to(torch.int32)
        self.uniforms = rand(n, k + -(-V // BLOCK) + 1, dtype=torch.float64)

    def call(self, e3, **more):
        return e3.e3_verify_drafts(self.logits, self.temps, self.draft_tok, self.uniforms, draft_len=self.draft_len,
                                   draft_logits=self.draft_logits, draft_temps=self.draft_temps, draft_logp=self.draft_logp, **more)

    def check(self, e3, **more):
        got = self.call(e3, **more)
        want = reference(self)
        tok, kept, logp, ent = (x.cpu().numpy() for x in got)
        assert np.array_equal(kept, want[1]), (kept, want[1])
        assert np.array_equal(tok, want[0]), np.argwhere(tok != want[0])[:5]
        # fp32 sums of the normaliser are good to 1e-5 of it at the very most, and so are the logarithms, absolutely
        assert_close("logp", logp, want[2], 1e-5)
        assert_close("ent", ent, want[3], 1e-5)
        return got


def host(x):
    return None if x is None else x.detach().float().cpu().numpy().astype(np.float64) if x.is_floating_point() and x.dtype != torch.float64 else x.cpu().numpy()


def probabilities(z, tau):
    """softmax(z / tau), its logarithm and its entropy; None for a row that cannot be used."""
    if not (tau >= 0 and tau < INF) or np.isnan(z).any() or (z == INF).any() or (z == -INF).all():
        return None
    if tau == 0:
        p = np.zeros_like(z)
        p[int(np.argmax(z))] = 1.0
        return p, np.where(p > 0, 0.0, -INF), 0.0
    x = z / tau
    x = x - x.max()
    w = np.exp(x)
    lp = x - math.log(w.sum())
    p = np.exp(lp)
    return p, lp, float(-(p[p > 0] * lp[p > 0]).sum())


def reference(s):
    n, k, V = s.n, s.k, s.V
    z, y, u = host(s.logits).reshape(n, k + 1, V), host(s.draft_logits), host(s.uniforms)
    temps, drafts = host(s.temps), host(s.draft_tok)
    draft_temps = host(s.draft_temps) if s.draft_temps is not None else temps
    lens = np.clip(host(s.draft_len), 0, k) if s.draft_len is not None else np.full(n, k)
    tok, kept = np.full((n, k + 1), -1, np.int32), np.zeros(n, np.int32)
    logp, ent = np.zeros((n, k + 1)), np.zeros((n, k + 1))
    for b in range(n):
        for j in range(lens[b] + 1):
            row = probabilities(z[b, j], temps[b])
            uniform = u[b, j] if j < lens[b] else 0.0
            if row is None or not 0 <= uniform < 1:
                logp[b, j] = ent[b, j] = math.nan
                break
            p, lp, h = row
            left = p
            if j < lens[b]:
                d, q = drafts[b, j], None
                if 0 <= d < V:
                    if y is None or draft_temps[b] == 0:
                        q = np.zeros(V)
                        q[d] = 1.0
                    else:
                        yr, lq, t = y[b * k + j], float(host(s.draft_logp)[b, j]), draft_temps[b]
                        if 0 < t < INF and np.isfinite(yr[d]) and lq < 1:
                            with np.errstate(invalid="ignore", over="ignore"):
                                q = np.exp((yr - yr[d]) / t + lq)
                if q is not None and uniform * q[d] < p[d]:
                    tok[b, j], logp[b, j], ent[b, j] = d, lp[d], h
                    kept[b] += 1
                    continue
                if q is not None:
                    left = np.where(p > q, p - q, 0.0)  # (NaN: nothing is left)
                    if left.sum() == 0:
                        left = p
            v = u[b, k:-1]
            if temps[b] > 0 and not ((v >= 0) & (v < 1) & (u[b, -1] >= 0) & (u[b, -1] < 1)).all():
                logp[b, j] = ent[b, j] = math.nan
                break
            if temps[b] == 0:
                t = int(np.argmax(p))
            else:
                full = np.zeros(len(v) * BLOCK)
                full[:V] = left
                sums = full.reshape(-1, BLOCK).sum(1)
                with np.errstate(divide="ignore"):
                    score = np.where(sums > 0, np.log(sums) - np.log(-np.log(v)), -INF)
                block = int(np.argmax(score))
                part = full[block * BLOCK:(block + 1) * BLOCK]
                above = np.flatnonzero((np.cumsum(part) > u[b, -1] * part.sum()) & (part > 0))
                t = block * BLOCK + (int(above[0]) if len(above) else int(np.flatnonzero(part)[-1]))
            tok[b, j], logp[b, j], ent[b, j] = t, lp[t], h
            break
    return tok, kept, logp, ent


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("model", [True, False])
@pytest.mark.parametrize("n, k, V", [(1, 1, 1), (2, 3, 2), (3, 1, 255), (3, 2, 256), (5, 4, 257), (40, 2, 1000), (2, 8, 20011), (9, 3, 33333), (700, 1, 300),
                                     (3, 2, 70001)])
def test_against_the_definition(e3, dtype, model, n, k, V):
    Batch(n + k + V, n, k, V, dtype, model).check(e3)
    Batch(n * k + V, n, k, V, dtype, model, ragged=True, greedy=0.3).check(e3)


@pytest.mark.parametrize("n, k, V", [(1, 4, 151936), (60, 3, 9000)])
def test_longer_rows_and_many_sequences(e3, n, k, V):
    for model in (True, False):
        Batch(V, n, k, V, torch.bfloat16, model).check(e3)


@pytest.mark.parametrize("dtype, V", [(torch.float32, 700003), (torch.bfloat16, 1500001)])
def test_rows_longer_than_the_shared_memory_of_their_blocks(e3, dtype, V):
    for model in (True, False):
        Batch(V, 2, 1, V, dtype, model).check(e3)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_no_drafts_is_a_draw_from_the_target(e3, dtype):
    s = Batch(1, 6, 0, 5000, dtype, model=False)
    s.check(e3)


def test_strides(e3):
    for off in (0, 1, 2, 3):
        for dtype in (torch.float32, torch.bfloat16):
            s = Batch(off, 4, 2, 700, dtype)
            wide = torch.zeros((12, 720), device="cuda", dtype=dtype)
            wide[:, off:off + 700] = s.logits
            wide[:, :off], wide[:, off + 700:] = float("nan"), float("nan")  # what lies around the rows is not looked at
            s.logits = wide[:, off:off + 700]
            wide = torch.full((8, 711), float("nan"), device="cuda", dtype=dtype)
            wide[:, off:off + 700] = s.draft_logits
            s.draft_logits = wide[:, off:off + 700]
            wide = torch.full((4, 20), 5.0, device="cuda", dtype=torch.float64)
            wide[:, 3:3 + s.uniforms.shape[1]] = s.uniforms
            s.uniforms = wide[:, 3:3 + s.uniforms.shape[1]]
            s.check(e3)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("fill", [-INF, -1e9, "lowest"])
def test_masked_vocabulary(e3, dtype, fill):
    fill = torch.finfo(dtype).min if fill == "lowest" else fill
    for model in (True, False):
        s = Batch(3, 8, 2, 3001, dtype, model)
        s.logits[:, 5::3] = fill
        s.logits[1], s.logits[4] = fill, fill
        s.logits[4, 77] = 1.0
        if fill != -INF:
            s.logits[2, :] = fill  # nothing but the fill value: uniform
        if model:
            s.draft_logits[3:9, 7::2] = fill
            s.draft_logp = (s.draft_logits.double() / s.draft_temps.double().repeat_interleave(2)[:, None]).log_softmax(-1).gather(
                1, s.draft_tok.view(-1, 1).long()).view(8, 2).float()
            s.draft_logp.nan_to_num_(nan=-1.0)
        s.check(e3)


def test_rows_and_uniforms_that_cannot_be_used(e3):
    s = Batch(4, 12, 2, 900, greedy=0.2)
    s.logits[0, 5] = float("nan")       # sequence 0, first position
    s.logits[3 * 1 + 1, 899] = INF      # sequence 1, second position, if it is reached
    s.logits[3 * 2] = -INF
    s.temps[3], s.temps[4], s.temps[5] = -1.0, float("nan"), INF
    s.uniforms[6, 0], s.uniforms[7, 1], s.uniforms[8, 3], s.uniforms[9, -1], s.uniforms[10, 0] = 1.0, -0.1, float("nan"), 1.5, float("nan")
    s.check(e3)


def test_drafts_that_cannot_be_used(e3):
    s = Batch(5, 10, 2, 900)
    s.draft_tok[0, 0], s.draft_tok[1, 1], s.draft_tok[2, 0] = -1, 900, 2 ** 31 - 1
    s.draft_logp[3, 0], s.draft_logp[4, 0] = float("nan"), INF
    s.draft_temps[5], s.draft_temps[6], s.draft_temps[7] = 0.0, -1.0, float("nan")
    s.draft_logits[2 * 8, int(s.draft_tok[8, 0])] = -INF
    s.draft_logits[2 * 9, 100:200], s.draft_logits[2 * 9, 300] = float("nan"), INF  # entries that are not drawn
    s.uniforms[:, 0] = 0.999
    s.check(e3)
    s = Batch(6, 5, 3, 500, ragged=True)
    s.draft_len = torch.tensor([-4, 0, 7, 3, 2 ** 31 - 1], device="cuda", dtype=torch.int32)
    s.check(e3)


def test_uniforms_of_zero(e3):
    s = Batch(7, 6, 2, 2000)
    s.uniforms[0] = 0.0
    s.uniforms[1, :2], s.uniforms[2, 2:-1], s.uniforms[3, -1] = 0.0, 0.0, 0.0
    s.uniforms[2, 5] = 1e-300
    got = s.call(e3)
    want = reference(s)
    assert torch.equal(got[1].cpu(), torch.from_numpy(want[1]))
    some = [1, 2, 3, 4, 5]  # (where every block has the uniform 0 no block leads)
    assert np.array_equal(got[0].cpu().numpy()[some], want[0][some])


def test_equal_distributions_keep_every_draft(e3):
    """p = q: u q < p wherever the draft's normaliser does not round up, and nothing is left where it does."""
    s = Batch(8, 30, 3, 4000, error=0.0)
    s.uniforms[:, :3] = 0.999
    s.check(e3)
    s.draft_logp = s.draft_logp + 1.0  # (a normaliser that is off: q > p everywhere, so a refusal draws from p)
    s.draft_logp.clamp_max_(0.9)
    s.uniforms[:, 0] = 0.99
    s.check(e3)


@pytest.mark.parametrize("sign", [-1, 1])
def test_uniforms_next_to_the_ratio(e3, sign):
    """Closer to p / q than sums in fp32 can tell."""
    for model in (True, False):
        s = Batch(9, 20, 1, 3000, model=model)
        for b in range(20):
            p = probabilities(host(s.logits)[2 * b], float(s.temps[b]))[0][int(s.draft_tok[b, 0])]
            q = math.exp(float(s.draft_logp[b, 0])) if model else 1.0
            if p < q:
                s.uniforms[b, 0] = p / q * (1 + sign * 1e-9 * (b + 1))
        s.check(e3)


# gaps that need the row's normaliser in fp64, that scores in fp64 settle without it, and that fp32 settles
@pytest.mark.parametrize("gap", [s * g for g in (1e-9, 1e-7, 1e-6, 1e-5, 1e-4) for s in (-1, 1)])
def test_blocks_and_entries_next_to_each_other(e3, gap):
    """Two leading blocks, and a prefix sum and the uniform, close to each other."""
    for model in (True, False):
        s = Batch(10, 12, 1, 2800, model=model)
        s.uniforms[:, 0] = 1 - 1e-12  # refused nearly everywhere
        tok, kept, _, _ = reference(s)
        z, u = host(s.logits), host(s.uniforms)
        for b in range(12):
            a = int(kept[b])
            p = probabilities(z[2 * b + a], float(s.temps[b]))[0]
            if a == 0:
                d = int(s.draft_tok[b, 0])
                if model:
                    y = host(s.draft_logits)[b]
                    p = np.maximum(p - np.exp((y - y[d]) / float(s.draft_temps[b]) + float(s.draft_logp[b, 0])), 0)
                else:
                    p[d] = 0
            full = np.zeros(11 * BLOCK)
            full[:2800] = p
            sums = full.reshape(-1, BLOCK).sum(1)
            score = np.log(sums) - np.log(-np.log(u[b, 1:-1]))
            first, second = np.argsort(-score)[:2]
            if b % 2 == 0:  # the second block's uniform puts it next to the first
                s.uniforms[b, 1 + second] = math.exp(-math.exp(-(score[first] + gap - math.log(sums[second]))))
            else:  # the draw inside the block next to a border
                part = full[first * BLOCK:(first + 1) * BLOCK]
                prefix = np.cumsum(part) / part.sum()
                s.uniforms[b, -1] = min(max(prefix[100] * (1 + gap), 0.0), 1 - 1e-9)
        s.check(e3)


def test_a_rare_block_next_to_a_confident_one(e3):
    """A row whose best token has all but 5e-5 of the mass, and a block of those 5e-5 whose uniform brings it next to the best token's."""
    deltas = [d * s for d in (1e-7, 1e-6, 3e-6, 1e-5) for s in (1, -1)]
    for far in (-9.5, -9.9, -10.4):
        s = Batch(21, len(deltas), 0, 64 * BLOCK)
        s.draft_logits = s.draft_temps = s.draft_logp = None
        s.logits.fill_(-300.0)
        s.logits[:, 5], s.logits[:, 32 * BLOCK + 7] = 0.0, far
        s.temps.fill_(1.0)
        s.uniforms.fill_(0.5)
        s.uniforms[:, 0] = math.exp(-1.0)  # (a variate of zero)
        for b, delta in enumerate(deltas):
            s.uniforms[b, 32] = math.exp(-math.exp(float(np.float32(far)) + delta))
        tok = s.check(e3)[0].cpu().numpy()[:, 0]
        assert [int(t) for t in tok] == [5 if d > 0 else 32 * BLOCK + 7 for d in deltas]


def test_outputs_given_and_left_out(e3):
    s = Batch(11, 5, 2, 600)
    tok, kept, logp, ent = s.call(e3)
    out = [torch.full_like(x, 3) for x in (tok, kept, logp, ent)]
    got = s.call(e3, out_tok=out[0], out_kept=out[1], out_logp=out[2], out_ent=out[3], workspace=torch.empty(1 << 16, dtype=torch.uint8, device="cuda"))
    assert all(x is y for x, y in zip(got, out)) and all(torch.equal(x, y) for x, y in zip(out, (tok, kept, logp, ent)))
    got = s.call(e3, want_logp=False, want_ent=False)
    assert got[2] is None and got[3] is None and torch.equal(got[0], tok) and torch.equal(got[1], kept)


def test_the_workspace_may_hold_anything(e3):
    s = Batch(12, 7, 3, 5000)
    want = s.call(e3)
    for fill in (0, 255, 1):
        ws = torch.full((e3.e3_workspace_bytes(e3.E3_CALL_VERIFY_DRAFTS, 28, 5000),), fill, dtype=torch.uint8, device="cuda")
        assert all(torch.equal(x, y) for x, y in zip(s.call(e3, workspace=ws), want))


def test_graphs_and_streams(e3):
    s, t = Batch(13, 6, 2, 9000, torch.bfloat16), Batch(14, 9, 3, 9000, torch.bfloat16)
    want, other_want = s.call(e3), t.call(e3)
    graphs, outs = [], []
    for x in (s, t):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(x.call(e3))
        graphs.append(g)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        for o in outs:
            for x in o:
                x.fill_(9)
        torch.cuda.synchronize()
        graphs[0].replay()
        with torch.cuda.stream(other):
            graphs[1].replay()
            there = s.call(e3, stream=other)
        here = t.call(e3)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(outs[0], want)) and all(torch.equal(x, y) for x, y in zip(outs[1], other_want))
        assert all(torch.equal(x, y) for x, y in zip(there, want)) and all(torch.equal(x, y) for x, y in zip(here, other_want))


@pytest.mark.parametrize("model", [True, False])
def test_tokens_are_distributed_like_the_target(e3, model):
    """The first emitted token of many sequences with the same rows: chi-square against p (a constant of the test: the seed is fixed)."""
    n, V = 40000, 300
    s = Batch(15, 1, 1, V, model=model, sharp=1.5, error=1.0)
    one = Batch(16, n, 1, V, model=False)  # (its uniforms)
    s.n, s.uniforms = n, one.uniforms
    p = probabilities(host(s.logits)[0], float(s.temps[0]))[0]
    if model:
        q = probabilities(host(s.draft_logits)[0], float(s.draft_temps[0]))[0]
        drawn = np.random.default_rng(3).choice(V, n, p=q / q.sum())
        s.draft_tok = torch.from_numpy(drawn.astype(np.int32)).cuda().view(n, 1)
        s.draft_logp = torch.from_numpy(np.log(q[drawn]).astype(np.float32)).cuda().view(n, 1)
        s.draft_logits, s.draft_temps = s.draft_logits.expand(n, V).contiguous(), s.draft_temps.expand(n).contiguous()
    else:
        s.draft_tok = s.draft_tok.expand(n, 1).contiguous()
    s.logits, s.temps = s.logits.repeat(n, 1), s.temps.expand(n).contiguous()
    tok, kept, _, _ = s.call(e3)
    assert 0.1 < kept.float().mean().item() < 0.95 or not model
    count = np.bincount(tok[:, 0].cpu().numpy(), minlength=V)
    order = np.argsort(-p)
    bins, seen, expected = [], 0, 0.0
    for i in order:  # entries with few expected draws go together
        seen, expected = seen + count[i], expected + p[i] * n
        if expected >= 10:
            bins.append((seen, expected))
            seen, expected = 0, 0.0
    bins.append((seen, max(expected, 1e-9)))
    chi = sum((o - e) ** 2 / e for o, e in bins if e > 1)
    df = len(bins)
    assert chi < df + 5 * math.sqrt(2 * df), (chi, df)


def test_refusals(e3):
    s = Batch(17, 3, 2, 400)
    s.check(e3)
    for name, bad in [("logits", s.logits[:8]), ("logits", s.logits.half()), ("temps", s.temps[:2]), ("temps", s.temps.double()),
                      ("draft_tok", s.draft_tok.long()), ("draft_tok", s.draft_tok.view(-1)), ("uniforms", s.uniforms.float()),
                      ("uniforms", s.uniforms[:, 1:]), ("draft_logits", s.draft_logits[:5]), ("draft_logits", s.draft_logits.bfloat16()),
                      ("draft_logp", s.draft_logp.double()), ("draft_temps", s.draft_temps[:1]), ("temps", s.temps.cpu()),
                      ("draft_len", torch.zeros(3, device="cuda"))]:
        t = Batch(17, 3, 2, 400)
        setattr(t, name, bad)
        with pytest.raises(ValueError):
            t.call(e3)
    for out in ("out_tok", "out_kept", "out_logp", "out_ent"):
        with pytest.raises(ValueError):
            s.call(e3, **{out: torch.zeros((3, 2), device="cuda")})
    with pytest.raises(TypeError):
        e3.e3_verify_drafts(s.logits, s.temps, s.draft_tok, s.uniforms, draft_logits=s.draft_logits)
    with pytest.raises(e3.E3Error):
        s.call(e3, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
