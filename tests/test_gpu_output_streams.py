"""Calls with `stream=`: their outputs' memory is neither taken from work that is still under way elsewhere nor given away before the call has run."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def e3():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2505_18573_b200 import binding
    binding.lib()
    return binding


def calls(e3):
    """Name -> call(stream) -> an output of 1 to 2 MB, whose memory comes from the allocator's pool of larger blocks."""
    f = lambda *s: torch.full(s, 0.25, device="cuda")  # noqa: E731
    n = 400_000
    logits, temps, tok = f(n, 4), f(n), torch.zeros(n, device="cuda", dtype=torch.int32)
    logp, ent = e3.e3_token_logp_entropy(logits, tok)[:2]
    upstream = f(100_000)
    rewards, off = f(n), torch.arange(0, n + 1, 8, device="cuda")
    u = torch.full((n, 2), 0.5, device="cuda", dtype=torch.float64)
    none = torch.empty((n, 0), device="cuda", dtype=torch.int32)
    table, few = f(300, 1024), torch.zeros(400, device="cuda", dtype=torch.int32)
    q, sq = e3.e3_quantize(f(400, 256))
    w, sw = e3.e3_quantize(f(2000, 256), 128)
    return {
        "e3_sample": lambda s: e3.e3_sample(logits, temps, 1, 0, stream=s)[0],
        "e3_token_logp_entropy": lambda s: e3.e3_token_logp_entropy(logits, tok, stream=s)[0],
        "e3_token_logp_entropy_backward": lambda s: e3.e3_token_logp_entropy_backward(logits[:100_000], tok[:100_000], logp[:100_000], ent[:100_000], upstream, stream=s),
        "e3_group_advantage": lambda s: e3.e3_group_advantage(rewards, off, stream=s)[0],
        "e3_verify_drafts": lambda s: e3.e3_verify_drafts(logits, temps, none, u, stream=s)[0],
        "e3_embed_tokens": lambda s: e3.e3_embed_tokens(table, few, stream=s),
        "e3_embed_tokens_backward": lambda s: e3.e3_embed_tokens_backward(table, few[:300], 300, stream=s),
        "e3_quantize": lambda s: e3.e3_quantize(logits.view(1000, 1600), stream=s)[0],
        "e3_project_vocab": lambda s: e3.e3_project_vocab(q, sq, w, sw, stream=s),
    }


def ready(e3, name):
    """(call, its output, another stream): all inputs are there, and the other stream has its workspace."""
    call, other = calls(e3)[name], torch.cuda.Stream()
    torch.cuda.synchronize()
    want = call(None)
    torch.cuda.synchronize()
    call(other)
    torch.cuda.synchronize()
    return call, want, other


NAMES = ("e3_sample", "e3_token_logp_entropy", "e3_token_logp_entropy_backward", "e3_group_advantage", "e3_verify_drafts", "e3_embed_tokens",
         "e3_embed_tokens_backward", "e3_quantize", "e3_project_vocab")


@pytest.mark.parametrize("name", NAMES)
def test_outputs_dropped_before_the_call_has_run(e3, name):
    call, want, other = ready(e3, name)
    size = want.numel() * want.element_size()
    with torch.cuda.stream(other):
        torch.cuda._sleep(100_000_000)  # some 50 ms
    out = call(other)
    del out
    fresh = [torch.full((size,), 7, device="cuda", dtype=torch.uint8) for _ in range(3)]
    torch.cuda.synchronize()
    assert all(bool((x == 7).all()) for x in fresh)


@pytest.mark.parametrize("name", NAMES)
def test_memory_that_the_current_stream_still_reads(e3, name):
    call, want, other = ready(e3, name)
    size = want.numel() * want.element_size()
    kept = [torch.empty(size, device="cuda", dtype=torch.uint8) for _ in range(3)]
    torch.cuda.synchronize()
    read = [torch.full((size,), 7, device="cuda", dtype=torch.uint8) for _ in range(3)]
    torch.cuda.synchronize()
    torch.cuda._sleep(100_000_000)
    for x, y in zip(kept, read):
        x.copy_(y)
    del read, y
    got = call(other)
    torch.cuda.synchronize()
    assert all(bool((x == 7).all()) for x in kept)
    assert torch.equal(got.view(torch.uint8), want.view(torch.uint8))


@pytest.mark.parametrize("name", NAMES)
def test_outputs_that_the_current_stream_still_reads(e3, name):
    """Dropped with a read under way in the current stream, which has waited for the call: the next call in the other stream gets other memory."""
    call, want, other = ready(e3, name)
    copy = torch.empty_like(want)
    out = call(other)
    torch.cuda.current_stream().wait_stream(other)
    torch.cuda._sleep(100_000_000)
    copy.view(torch.uint8).copy_(out.view(torch.uint8))
    del out
    with torch.cuda.stream(other):
        fresh = [torch.full_like(want.view(torch.uint8), 7) for _ in range(3)]
    torch.cuda.synchronize()
    assert torch.equal(copy.view(torch.uint8), want.view(torch.uint8)) and len(fresh) == 3


@pytest.mark.parametrize("name", NAMES)
def test_a_stream_that_joins_a_capture(e3, name):
    """Captured through a second stream that the capture forks to, replayed twice, its output dropped last."""
    call, want, other = ready(e3, name)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        here = torch.cuda.current_stream()
        other.wait_stream(here)
        out = call(other)
        here.wait_stream(other)
        copy = out.clone()
    for _ in range(2):
        out.view(torch.uint8).zero_()
        copy.view(torch.uint8).zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(copy.view(torch.uint8), want.view(torch.uint8))
    del out, copy
    assert torch.full((1000,), 3, device="cuda").eq(3).all()
