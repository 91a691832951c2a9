"""Calls of the operators at both ends of the vocabulary that their contracts allow and that are seldom made."""
import pytest
import torch

from test_gpu_embed import exact_gradient, generator, rounded_to, tokens
from test_gpu_far_rows import apart
from test_gpu_verify import Batch, reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def e3():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2505_18573_b200 import binding
    binding.lib()
    return binding


def test_gradient_of_no_tokens_into_rows_far_apart(e3):
    """Zeroed, whatever the distance of its rows; what lies between them is left alone."""
    keep = []
    for dtype in (torch.bfloat16, torch.float32):
        table = apart(torch.full((5, 70), 3.0, device="cuda", dtype=dtype), keep, off=1)
        between = [keep[-1].as_strided((5,), (table.stride(0),), o) for o in (0, 71)]
        for x in between:
            x.fill_(7.0)
        none = torch.zeros((0, 70), device="cuda", dtype=dtype)
        e3.e3_embed_tokens_backward(none, torch.zeros(0, device="cuda", dtype=torch.int32), 5, out=table)
        assert bool((table == 0).all()) and all(bool((x == 7).all()) for x in between)
        keep.clear()


def test_shapes_of_tokens(e3):
    table = torch.randn((50, 24), generator=generator(1), device="cuda")
    one = torch.tensor(7, device="cuda", dtype=torch.int32)
    assert torch.equal(e3.e3_embed_tokens(table, one), table[7])
    assert e3.e3_embed_tokens(table, torch.zeros((3, 0, 2), device="cuda", dtype=torch.int32)).shape == (3, 0, 2, 24)
    assert torch.equal(e3.e3_embed_tokens(table, torch.arange(24, device="cuda", dtype=torch.int32).view(2, 3, 4)), table[:24].view(2, 3, 4, 24))


@pytest.mark.parametrize("table", [torch.float32, torch.bfloat16])
def test_wide_vectors(e3, table):
    """More columns than a CTA of the sums takes."""
    for n, D in ((700, 100_003), (5000, 40_000)):
        r = generator(D)
        g, tok = torch.randn((n, D), generator=r, device="cuda"), tokens(r, n, 300)
        got = e3.e3_embed_tokens_backward(g, tok, 300, dtype=table)
        rounded_to(got, *exact_gradient(g, tok, 300, 1.0))


def test_many_sequences_of_short_rows(e3):
    n, times = 4096, 366
    small = Batch(4, n, 1, 3)
    want = reference(small)
    for name in ("logits", "temps", "draft_tok", "draft_logits", "draft_temps", "draft_logp", "uniforms"):
        x = getattr(small, name)
        setattr(small, name, x.repeat(times, *([1] * (x.dim() - 1))))
    tok, kept, _, _ = small.call(e3)
    assert torch.equal(tok, torch.from_numpy(want[0]).cuda().repeat(times, 1)) and torch.equal(kept, torch.from_numpy(want[1]).cuda().repeat(times))


def test_every_operator_in_one_graph(e3):
    """Captured together, two graphs of different inputs replayed in turn: each its own workspaces."""
    r = generator(5)

    def inputs(seed, n):
        r.manual_seed(seed)
        return (torch.randn((500, 256), generator=r, device="cuda").bfloat16(), tokens(r, n, 500), torch.randn((n, 256), generator=r, device="cuda").bfloat16(),
                Batch(seed, 6, 2, 500, torch.bfloat16))

    def run(table, tok, g, s):
        hidden = e3.e3_embed_tokens(table, tok, 2.0)
        q, sq = e3.e3_quantize(hidden.view(-1, 256)[:300])
        w, sw = e3.e3_quantize(table, 128)
        return [hidden, e3.e3_project_vocab(q, sq, w, sw), e3.e3_embed_tokens_backward(g, tok, 500), *s.call(e3)]

    made = [inputs(1, 6000), inputs(2, 900)]
    want = [run(*x) for x in made]
    graphs, outs = [], []
    for x in made:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            outs.append(run(*x))
    for _ in range(3):
        for o in outs:
            for x in o:
                x.fill_(9)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert all(torch.equal(a.nan_to_num(5.0), b.nan_to_num(5.0)) for a, b in zip(o, w))
