"""Rows that lie further apart than 32 bits reach: every operator at both ends of the vocabulary against the same call on compact tensors."""
import pytest
import torch

from test_gpu_project import E4M3, operands
from test_gpu_verify import Batch

pytestmark = pytest.mark.gpu

FAR = (1 << 32) + (1 << 20)  # entries of a buffer


@pytest.fixture(scope="module")
def e3():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2505_18573_b200 import binding
    binding.lib()
    return binding


def apart(x, buffers, multiple=16, off=0):
    """x, its rows spread over a buffer of FAR entries of its type; `off` entries behind a 16-byte boundary."""
    buf = torch.empty(FAR, dtype=x.dtype, device="cuda")
    buffers.append(buf)
    stride = (FAR - x.shape[1] - off) // max(1, x.shape[0] - 1) // multiple * multiple
    view = buf[off:].as_strided(x.shape, (stride, 1))
    view.copy_(x)
    assert (x.shape[0] - 1) * stride > 1 << 31
    return view


def generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


@pytest.mark.parametrize("off", [0, 1])
@pytest.mark.parametrize("tokens", [40, 5000])
def test_embedding(e3, tokens, off):
    g, keep = generator(1), []
    table = torch.randn((700, 136), generator=g, device="cuda").bfloat16()
    tok = torch.randint(-1, 700, (tokens,), generator=g, device="cuda", dtype=torch.int32)
    want = e3.e3_embed_tokens(table, tok, 1.5)
    out = apart(torch.full_like(want, 7.0), keep, off=off)
    e3.e3_embed_tokens(apart(table, keep, off=off), tok, 1.5, out=out)
    assert torch.equal(out, want)
    want = e3.e3_embed_tokens_backward(out.contiguous(), tok, 700, 0.5)
    grad = apart(torch.full_like(table, 7.0), keep, off=off)
    e3.e3_embed_tokens_backward(out, tok, 700, 0.5, out=grad)
    assert torch.equal(grad, want)


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("off", [0, 1])
def test_quantize(e3, block_rows, off):
    x, keep = torch.randn((500, 300), generator=generator(2), device="cuda").bfloat16(), []
    want = e3.e3_quantize(x, block_rows)
    q = apart(torch.zeros((500, 300), dtype=E4M3, device="cuda"), keep, off=off)
    got = e3.e3_quantize(apart(x, keep, off=off), block_rows, out_q=q)
    assert torch.equal(q.view(torch.uint8), want[0].view(torch.uint8)) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("off", [0, 1])
@pytest.mark.parametrize("rows", [9, 100, 300])
def test_project(e3, rows, off):
    x, sx, w, sw = operands(3, rows, 600, 400)
    keep = []
    want = e3.e3_project_vocab(x, sx, w, sw)
    out = apart(torch.zeros_like(want), keep, off=off)
    e3.e3_project_vocab(apart(x, keep), apart(sx, keep), apart(w, keep), sw, out=out)
    assert torch.equal(out, want)


@pytest.mark.parametrize("off", [0, 1])
def test_verify(e3, off):
    s, keep = Batch(4, 40, 3, 1100, torch.bfloat16), []
    want = s.call(e3)
    s.logits, s.draft_logits = apart(s.logits, keep, off=off), apart(s.draft_logits, keep, off=off)
    got = s.call(e3)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    # (2,200 bytes to a row: the compact rows begin elsewhere within 16 bytes, and are added in another order; either is within 1e-5)
    for a, b in zip(got[2:], want[2:]):
        assert float((a - b).abs().max()) <= 2e-5


def test_many_drafts_of_a_sequence(e3):
    """More positions than a CTA has threads, and a draft that all of them keep."""
    s = Batch(5, 3, 300, 64, error=0.02)
    s.uniforms[0, :300] = 0.0
    s.check(e3)
