"""Embedding of tokens and the gradient of its table against sums in 64 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def e3():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2505_18573_b200 import binding
    binding.lib()
    return binding


def tokens(g, n, V, pad=0.1, hot=0.3):
    """Some tokens far more often than the others, some padding."""
    t = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int32)
    t = torch.where(torch.rand(n, generator=g, device="cuda") < hot, t % max(1, V // 50 + 1), t)
    return torch.where(torch.rand(n, generator=g, device="cuda") < pad, -1, t).to(torch.int32)


def generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def rounded_to(got, exact, terms_abs, count):
    """`got` is `exact` but for fp32 sums of `count` terms (of absolute sum terms_abs: a unit of 2^-24 each), two products and one rounding to its
    type (half a step)."""
    half = torch.finfo(got.dtype).eps / 2
    sums = terms_abs * (count + 2) * 2.0 ** -24
    err = (got.double() - exact).abs()
    bound = sums + (exact.abs() + sums) * half + 1e-30
    assert bool((err <= bound).all()), (err - bound).max()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("n, V, D", [(1, 1, 1), (3, 5, 7), (33, 100, 8), (257, 1000, 1001), (64, 40, 1536), (5, 9, 4097)])
def test_lookup(e3, dtype, n, V, D):
    g = generator(n + V)
    table = torch.randn((V, D), generator=g, device="cuda").to(DTYPES[dtype])
    tok = tokens(g, n, V)
    got = e3.e3_embed_tokens(table, tok, scale=1.7)
    scale = float(torch.tensor(1.7, dtype=torch.float32))
    want = torch.where((tok >= 0)[:, None], table.double()[tok.long().clamp_min(0)] * scale, 0.0)
    assert got.shape == (n, D) and got.dtype == table.dtype
    # a product in fp32 and one rounding
    assert bool(((got.double() - want).abs() <= want.abs() * (torch.finfo(got.dtype).eps / 2 + 2.0 ** -24)).all())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_lookup_through_strides_and_shapes(e3, dtype):
    g = generator(3)
    wide = torch.randn((50, 140), generator=g, device="cuda").to(DTYPES[dtype])
    tok = tokens(g, 24, 50).view(4, 6)
    for lo in (0, 1, 8):  # rows that begin on a vector and off it
        table = wide[:, lo:lo + 100]
        got = e3.e3_embed_tokens(table, tok)
        want = torch.where((tok >= 0)[..., None], table[tok.long().clamp_min(0)], 0.0).to(table.dtype)
        assert got.shape == (4, 6, 100) and torch.equal(got, want)
        out = torch.full((24, 120), 7.0, device="cuda", dtype=table.dtype)
        e3.e3_embed_tokens(table, tok.view(-1), out=out[:, 8:108])
        assert torch.equal(out[:, 8:108], want.view(24, 100)) and bool((out[:, :8] == 7).all()) and bool((out[:, 108:] == 7).all())


def test_lookup_of_tokens_outside_the_vocabulary(e3):
    table = torch.ones((5, 24), device="cuda", dtype=torch.bfloat16)
    got = e3.e3_embed_tokens(table, torch.tensor([4, 5, -1, -2, 2 ** 31 - 1, 0], device="cuda", dtype=torch.int32)).float()
    assert bool((got[[0, 5]] == 1).all()) and bool((got[2] == 0).all()) and bool(got[[1, 3, 4]].isnan().all())
    assert e3.e3_embed_tokens(table, torch.empty(0, device="cuda", dtype=torch.int32)).shape == (0, 24)


def exact_gradient(g, tok, V, scale):
    live = tok >= 0
    want = torch.zeros((V, g.shape[1]), device="cuda", dtype=torch.float64)
    size = torch.zeros_like(want)
    want.index_add_(0, tok[live].long(), g[live].double() * scale)
    size.index_add_(0, tok[live].long(), (g[live].double() * scale).abs())
    return want, size, torch.bincount(tok[live].long(), minlength=V)[:, None]


@pytest.mark.parametrize("dtype, table", [("fp32", "fp32"), ("bf16", "bf16"), ("bf16", "fp32"), ("fp32", "bf16")])
@pytest.mark.parametrize("n, V, D", [(1, 1, 1), (2, 3, 5), (31, 2, 8), (33, 1000, 64), (2049, 50, 1000), (4096, 70, 19), (4097, 70, 19), (129, 31, 2), (4000, 33, 1), (5000, 33333, 129),
                                     (4000, 70000, 4), (4097, 70000, 4), (300, 5001, 130), (5000, 5001, 130), (900, 1 << 22, 5), (1000, 2000, 300),
                                     (40000, 700, 72), (4097, 4097, 2056), (6000, 1 << 22, 3),
                                     (300000, 3000000, 8), (1200000, 5000, 16)])
def test_gradient(e3, dtype, table, n, V, D):
    r = generator(n + V + D)
    g = torch.randn((n, D), generator=r, device="cuda").to(DTYPES[dtype])
    tok = tokens(r, n, V)
    got = e3.e3_embed_tokens_backward(g, tok, V, scale=0.37, dtype=DTYPES[table])
    scale = float(torch.tensor(0.37, dtype=torch.float32))
    want, size, count = exact_gradient(g, tok, V, scale)
    assert got.shape == (V, D) and got.dtype == DTYPES[table]
    rounded_to(got, want, size, count)
    assert torch.equal(got, e3.e3_embed_tokens_backward(g, tok, V, scale=0.37, dtype=DTYPES[table]))  # a fixed order
    # added to what is there: rows of tokens that do not occur keep their bits
    before = torch.randn((V, D), generator=r, device="cuda").to(DTYPES[table])
    added = before.clone()
    assert e3.e3_embed_tokens_backward(g, tok, V, scale=0.37, out=added, accumulate=True) is added
    rounded_to(added, want + before.double(), size + before.double().abs(), count)
    absent = (count == 0).view(-1)
    assert torch.equal(added[absent], before[absent])


def test_gradient_of_one_hot_token(e3):
    """All tokens alike: one run over every segment."""
    for n in (31, 32, 33, 64, 128, 129, 4096, 4097, 5000, 40000):
        g = torch.randn((n, 40), generator=generator(n), device="cuda")
        got = e3.e3_embed_tokens_backward(g, torch.full((n,), 3, device="cuda", dtype=torch.int32), 5)
        want, size, count = exact_gradient(g, torch.full((n,), 3, device="cuda"), 5, 1.0)
        rounded_to(got, want, size, count)


def test_gradient_of_padding_alone_and_of_no_tokens(e3):
    for n in (0, 1, 700, 6000):
        tok = torch.full((n,), -1, device="cuda", dtype=torch.int32)
        tok[::2] = 99  # outside the vocabulary
        got = e3.e3_embed_tokens_backward(torch.ones((n, 12), device="cuda"), tok, 9, out=torch.full((9, 12), 5.0, device="cuda"))
        assert bool((got == 0).all())
        kept = e3.e3_embed_tokens_backward(torch.ones((n, 12), device="cuda"), tok, 9, out=torch.full((9, 12), 5.0, device="cuda"), accumulate=True)
        assert bool((kept == 5).all())


def test_gradient_through_strides(e3):
    r = generator(8)
    for lo in (0, 1, 4):
        g = torch.randn((300, 80), generator=r, device="cuda")[:, lo:lo + 64]
        tok = tokens(r, 300, 40)
        out = torch.full((40, 100), 7.0, device="cuda")
        e3.e3_embed_tokens_backward(g, tok, 40, out=out[:, 16:80])
        want, size, count = exact_gradient(g, tok, 40, 1.0)
        rounded_to(out[:, 16:80], want, size, count)
        assert bool((out[:, :16] == 7).all()) and bool((out[:, 80:] == 7).all())


def test_gradient_is_that_of_the_lookup(e3):
    """Differences of L = sum(w * lookup) along a direction of the table; the lookup is linear, so they are exact up to rounding."""
    r = generator(5)
    table, step, w = (torch.randn(s, generator=r, device="cuda") for s in ((60, 33), (60, 33), (500, 33)))
    tok = tokens(r, 500, 60)
    loss = lambda t: (w.double() * e3.e3_embed_tokens(t, tok, scale=2.0).double()).sum()  # noqa: E731
    slope = (loss(table + 0.5 * step) - loss(table - 0.5 * step)).item()
    grad = e3.e3_embed_tokens_backward(w, tok, 60, scale=2.0)
    along = (grad.double() * step.double()).sum().item()
    # two tables of one sum and one product, each of three roundings of 2^-24; the gradient's sums and product
    _, size, count = exact_gradient(w, tok, 60, 2.0)
    live = (tok >= 0)[:, None]
    entries = torch.where(live, (table.abs() + step.abs())[tok.long().clamp_min(0)], 0.0).double()
    bound = 2.0 ** -24 * (6 * (w.double().abs() * 2.0 * entries).sum() + ((count + 3) * size * step.double().abs()).sum())
    assert abs(slope - along) <= bound.item()


def test_gradient_in_a_graph_and_on_another_stream(e3):
    r = generator(6)
    g, tok = torch.randn((3000, 64), generator=r, device="cuda"), tokens(r, 3000, 500)
    want = e3.e3_embed_tokens_backward(g, tok, 500)
    out = torch.empty_like(want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        e3.e3_embed_tokens_backward(g, tok, 500, out=out)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        out.fill_(float("nan"))
        graph.replay()
        there = e3.e3_embed_tokens_backward(g, tok, 500, stream=other)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(there, want)


def test_refusals(e3):
    g, tok = torch.ones((4, 8), device="cuda"), torch.zeros(4, device="cuda", dtype=torch.int32)
    for call in (lambda: e3.e3_embed_tokens(g.half(), tok), lambda: e3.e3_embed_tokens(g, tok.long()), lambda: e3.e3_embed_tokens(g.t(), tok),
                 lambda: e3.e3_embed_tokens(g, tok.cpu()), lambda: e3.e3_embed_tokens(g, tok, out=g[:3]),
                 lambda: e3.e3_embed_tokens_backward(g, tok[:3], 9), lambda: e3.e3_embed_tokens_backward(g, tok, 9, accumulate=True),
                 lambda: e3.e3_embed_tokens_backward(g, tok, 9, dtype=torch.float16),
                 lambda: e3.e3_embed_tokens_backward(g, tok, 9, out=torch.zeros((8, 8), device="cuda"))):
        with pytest.raises(ValueError):
            call()
    for V in (0, -3, (1 << 22) + 1):
        with pytest.raises(e3.E3Error):
            e3.e3_embed_tokens_backward(g[:, :1], tok, V)
