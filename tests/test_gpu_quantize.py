"""8-bit values with a scale per block against the definition, worked out in 64 bits."""
import math

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


def reference(x, block_rows):
    """(q, scale): the smallest power of two s with max|x| <= 448 s, x / s to four significant bits (steps no finer than 2^-9), half to even."""
    x = x.double().cpu()
    rows, cols = x.shape
    q = torch.empty_like(x)
    scale = torch.empty((-(-rows // block_rows), -(-cols // 128)), dtype=torch.float64)
    for i in range(scale.shape[0]):
        for j in range(scale.shape[1]):
            at = (slice(i * block_rows, (i + 1) * block_rows), slice(j * 128, (j + 1) * 128))
            most = x[at].abs().max().item()
            if not math.isfinite(most) or x[at].isnan().any():
                scale[i, j], q[at] = math.nan, math.nan
                continue
            e = 0
            if most > 0:
                e = math.frexp(most / 448.0)[1] - 1
                e += most > 448.0 * 2.0 ** e
                e = max(e, -126)
            scale[i, j] = 2.0 ** e
            t = x[at] / 2.0 ** e
            step = torch.exp2(torch.floor(torch.log2(t.abs().clamp_min(2.0 ** -6))) - 3)
            q[at] = torch.round(t / step) * step
    return q, scale


def check(e3, x, block_rows):
    q, scale = e3.e3_quantize(x, block_rows)
    want_q, want_scale = reference(x, block_rows)
    assert q.dtype == torch.float8_e4m3fn and q.shape == x.shape and q.stride(0) % 16 == 0
    got = q.float().cpu().double()
    assert torch.equal(scale.cpu().double().nan_to_num(-1.0), want_scale.nan_to_num(-1.0))
    assert torch.equal(got.isnan(), want_q.isnan()) and torch.equal(got.nan_to_num(0.0), want_q.nan_to_num(0.0))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("rows, cols", [(1, 1), (3, 7), (2, 128), (5, 129), (127, 256), (128, 128), (129, 1000), (300, 136)])
def test_values_and_scales(e3, dtype, block_rows, rows, cols):
    g = torch.Generator(device="cuda")
    g.manual_seed(rows * 1000 + cols)
    x = torch.randn((rows, cols), generator=g, device="cuda") * torch.exp(4 * torch.randn((rows, 1), generator=g, device="cuda"))
    check(e3, x.to(dtype), block_rows)


@pytest.mark.parametrize("block_rows", [1, 128])
def test_ties_borders_and_sizes(e3, block_rows):
    # midpoints of neighbouring values, the largest value and just above it, subnormal results
    x = torch.zeros((8, 256), device="cuda")
    x[0, :40] = (torch.arange(40, device="cuda") + 0.5) * 8
    x[0, 40] = 448.0
    x[1, :3] = torch.tensor([448.0, 447.99, 1e-3], device="cuda")
    x[2, :3] = torch.tensor([448.0001, -464.0, 2.0 ** -9], device="cuda")
    x[3, :4] = torch.tensor([1e38, -3.4e38, 1.0, 0.0], device="cuda")
    x[4, 130:134] = torch.tensor([1e-38, 1e-40, -1e-45, 0.0], device="cuda")
    x[6, :2] = torch.tensor([-1.75, 1.7500001], device="cuda")
    for row in range(8):
        check(e3, x[row:row + 1], block_rows)
    check(e3, x, block_rows)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_nan_and_infinities_mark_their_block(e3, dtype, block_rows):
    x = torch.ones((130, 300), device="cuda", dtype=dtype)
    x[3, 5] = float("nan")
    x[4, 299] = float("inf")
    x[129, 130] = -float("inf")
    check(e3, x, block_rows)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_strides(e3, dtype, block_rows):
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    wide = torch.randn((140, 320), generator=g, device="cuda").to(dtype)
    for lo in (0, 1, 8):
        x = wide[:, lo:lo + 300]
        want_q, want_scale = e3.e3_quantize(x.contiguous(), block_rows)
        q = torch.zeros((140, 333), device="cuda").to(torch.float8_e4m3fn)
        got, scale = e3.e3_quantize(x, block_rows, out_q=q[:, 2:302])
        assert torch.equal(got.float(), want_q.float()) and torch.equal(scale, want_scale)
        assert bool((q[:, :2].float() == 0).all()) and bool((q[:, 302:].float() == 0).all())


def test_refusals(e3):
    x = torch.ones((4, 130), device="cuda")
    for call in (lambda: e3.e3_quantize(x, 2), lambda: e3.e3_quantize(x.half()), lambda: e3.e3_quantize(x.t()), lambda: e3.e3_quantize(x[0]),
                 lambda: e3.e3_quantize(x, out_q=torch.zeros((4, 130), device="cuda")), lambda: e3.e3_quantize(x.cpu()),
                 lambda: e3.e3_quantize(x, out_scale=torch.zeros((4, 1), device="cuda"))):
        with pytest.raises(ValueError):
            call()
    q, scale = e3.e3_quantize(x[:0])
    assert q.shape == (0, 130) and scale.shape == (0, 2)
