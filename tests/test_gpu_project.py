"""The projection in 8 bits against the same products in 64 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu

E4M3 = torch.float8_e4m3fn


@pytest.fixture(scope="module")
def e3():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    from paper_2505_18573_b200 import binding
    binding.lib()
    return binding


def eight_bits(g, rows, D, per, spread=1.0):
    """e4m3 values in rows padded to 16 bytes, the padding full of NaN, and fp32 scales that are no powers of two."""
    q = torch.full((rows, (D + 15) // 16 * 16), float("nan"), device="cuda").to(E4M3)
    q[:, :D] = (100 * torch.randn((rows, D), generator=g, device="cuda")).clamp(-448, 448).to(E4M3)
    scale = torch.exp(spread * torch.randn((-(-rows // per), -(-D // 128)), generator=g, device="cuda"))
    return q[:, :D], scale


def operands(seed, rows, V, D, spread=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (*eight_bits(g, rows, D, 1, spread), *eight_bits(g, V, D, 128, spread))


def values(q, scale, per):
    return q.double() * scale.double().repeat_interleave(per, 0)[:q.shape[0]].repeat_interleave(128, 1)[:, :q.shape[1]]


def check(e3, ops, dtype, out=None):
    x, sx, w, sw = ops
    got = e3.e3_project_vocab(x, sx, w, sw, dtype=dtype, out=out)
    a, b = values(x, sx, 1), values(w, sw, 128)
    want, size = a @ b.t(), a.abs() @ b.abs().t()
    assert got.shape == want.shape and got.dtype == dtype
    # sums of 128 exact products in 32 bits (each addition within 2^-23 of the sum of absolute values, as fp32 cut off rather than rounded would be),
    # a scale of two factors, a sum over the blocks; then one rounding to the type
    sums = size * (128 * 2.0 ** -23 + (sx.shape[1] + 3) * 2.0 ** -24)
    bound = sums + (want.abs() + sums) * torch.finfo(dtype).eps / 2 + 1e-30
    err = (got.double() - want).abs()
    assert bool((err <= bound).all()), (float((err - bound).max()), int((err > bound).sum()))
    return got


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows, V, D", [(1, 1, 1), (1, 128, 128), (3, 5, 17), (16, 129, 256), (17, 300, 100), (33, 1000, 384), (65, 257, 1000),
                                        (128, 640, 129), (129, 131, 300), (256, 1280, 512), (257, 999, 640), (600, 2500, 1024)])
def test_against_products_in_64_bits(e3, dtype, rows, V, D):
    check(e3, operands(rows + V + D, rows, V, D), dtype)


def test_one_entry_at_a_time_with_scales(e3):
    """Every scale in its place: one entry of each operand's row and block, the scales powers of two that differ from their neighbours'."""
    rows, V, D = 300, 520, 1100
    x, w = torch.zeros((rows, 1104), device="cuda"), torch.zeros((V, 1104), device="cuda")
    for blk in range(9):
        x[torch.arange(rows, device="cuda"), torch.minimum(torch.tensor(1099, device="cuda"), 128 * blk + torch.arange(rows, device="cuda") % 128)] = 1.0
        w[:, min(128 * blk + 5, 1099)] = 1.0
    x, w = x.to(E4M3)[:, :D], w.to(E4M3)[:, :D]
    sx = torch.exp2((torch.arange(rows, device="cuda")[:, None] * 3 + torch.arange(9, device="cuda")[None] * 5).remainder(11).float() - 5)
    sw = torch.exp2((torch.arange(5, device="cuda")[:, None] * 2 + torch.arange(9, device="cuda")[None] * 7).remainder(13).float() - 6)
    for dtype in (torch.float32, torch.bfloat16):
        got = e3.e3_project_vocab(x, sx, w, sw, dtype=dtype)
        assert torch.equal(got, (values(x, sx, 1) @ values(w, sw, 128).t()).to(dtype))


def test_scales_of_any_value(e3):
    """Zeros, negative and subnormal scales multiply like others; NaN reaches the rows and entries of its block and no others."""
    for rows in (40, 100, 200):
        for at, value in ((0, 0.0), (7, -2.0), (3, 1e-40), (5, 3.0)):
            for which in (1, 3):
                ops = operands(9, rows, 600, 500)
                ops[which].view(-1)[at] = value
                check(e3, ops, torch.float32)
        ops = operands(9, rows, 600, 500)
        ops[1][17, 2] = float("nan")
        ops[3][1, 0] = float("nan")
        got = e3.e3_project_vocab(*ops, dtype=torch.float32)
        nan = torch.zeros((rows, 600), dtype=torch.bool, device="cuda")
        nan[17] = True
        nan[:, 128:256] = True
        assert torch.equal(got.isnan(), nan)


def test_many_tiles_a_block(e3):
    """More tiles than SMs, so that the rings run on from tile to tile."""
    for rows in (1, 20, 40, 100, 300):
        check(e3, operands(rows, rows, 50000, 400), torch.bfloat16)


def test_one_entry_at_a_time(e3):
    """Every product in its place: one entry of the hidden states and one of the table each, all others zero."""
    for rows in (16, 32, 64, 128, 256):
        D, V = 300, 260
        x, w = torch.zeros((rows, 304), device="cuda"), torch.zeros((V, 304), device="cuda")
        at = torch.arange(rows, device="cuda")
        x[at, (7 * at) % D] = 1.0 + (at % 8) / 8
        w[torch.arange(V, device="cuda"), (3 * torch.arange(V, device="cuda")) % D] = 2.0
        x, w = x.to(E4M3)[:, :D], w.to(E4M3)[:, :D]
        ones = torch.ones((rows, 3), device="cuda"), torch.ones((3, 3), device="cuda")
        got = e3.e3_project_vocab(x, ones[0], w, ones[1], dtype=torch.float32)
        assert torch.equal(got, x.float() @ w.float().t())


def test_strides(e3):
    x, sx, w, sw = operands(5, 40, 700, 200)
    wide_x, wide_w = torch.full((40, 512), float("nan"), device="cuda").to(E4M3), torch.full((700, 256), float("nan"), device="cuda").to(E4M3)
    wide_x[:, 16:216], wide_w[:, 32:232] = x, w
    wide_sx, wide_sw = torch.full((40, 9), float("nan"), device="cuda"), torch.full((6, 5), float("nan"), device="cuda")
    wide_sx[:, 3:5], wide_sw[:, 1:3] = sx, sw
    want = check(e3, (x, sx, w, sw), torch.bfloat16)
    for off in (0, 1, 3):
        out = torch.full((40, 711), 7.0, device="cuda", dtype=torch.bfloat16)
        e3.e3_project_vocab(wide_x[:, 16:216], wide_sx[:, 3:5], wide_w[:, 32:232], wide_sw[:, 1:3], out=out[:, off:off + 700])
        assert torch.equal(out[:, off:off + 700], want) and bool((out[:, :off] == 7).all()) and bool((out[:, off + 700:] == 7).all())


def test_nan_and_extreme_scales(e3):
    x, sx, w, sw = operands(6, 20, 300, 300)
    sx[3, 1], sw[1, 2] = float("nan"), float("inf")
    x[5, 7] = float("nan")
    got = e3.e3_project_vocab(x, sx, w, sw, dtype=torch.float32)
    assert bool(got[3].isnan().all()) and bool(got[5].isnan().all())
    rest = [i for i in range(20) if i not in (3, 5)]
    assert bool(got[rest][:, :128].isfinite().all()) and not bool(got[rest][:, 128:256].isfinite().any()) and bool(got[rest][:, 256:].isfinite().all())
    check(e3, operands(7, 20, 300, 700, spread=10.0), torch.float32)


def test_from_hidden_states_to_logits(e3):
    """With e3_quantize: as near to the product of the unrounded matrices as the 8-bit values are to theirs (half a step of e4m3, 2^-4, each)."""
    g = torch.Generator(device="cuda")
    g.manual_seed(8)
    x, w = torch.randn((70, 512), generator=g, device="cuda").bfloat16(), torch.randn((1000, 512), generator=g, device="cuda").bfloat16()
    got = check(e3, (*e3.e3_quantize(x), *e3.e3_quantize(w, 128)), torch.float32)
    size = x.double().abs() @ w.double().abs().t()
    # (values below the smallest normal e4m3 number are off by half of 2^-9 of their scale, here at most 2^-10 * 2^-6 of the block's largest)
    assert bool(((got.double() - x.double() @ w.double().t()).abs() <= size * (2.0 ** -4 * 2 + 2.0 ** -8) + 512 * 6 * 6 * 2.0 ** -15).all())


def test_graphs_and_streams(e3):
    a, b = operands(9, 24, 5000, 500), operands(10, 200, 5000, 500)
    want = [e3.e3_project_vocab(*o) for o in (a, b)]
    graph, outs = torch.cuda.CUDAGraph(), []
    with torch.cuda.graph(graph):
        outs = [e3.e3_project_vocab(*o) for o in (a, b)]
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        for o in outs:
            o.fill_(float("nan"))
        graph.replay()
        there = [e3.e3_project_vocab(*o, stream=other) for o in (a, b)]
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(outs + there, want + want))


@pytest.mark.parametrize("rows, pairs", [(9, False), (100, False), (300, True)])
@pytest.mark.parametrize("block", [0, 6, 13])
def test_a_wait_that_runs_out(e3, rows, pairs, block):
    """A block whose copies never come: the call returns, the first thread block's unfinished logits read NaN, the status word tells."""
    ops = operands(12, rows, 150000, 512)  # more tiles than SMs or pairs of them, four blocks each
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    want = e3.e3_project_vocab(*ops, status=status)
    assert status.item() == 0
    e3.e3_test_arm_project_stall(block, 5_000_000)  # 5 ms instead of two seconds
    got = e3.e3_project_vocab(*ops, status=status)
    torch.cuda.synchronize()
    assert status.item() & e3.E3_STATUS_TIMEOUT
    bad = got.isnan()
    assert torch.equal(got[~bad], want[~bad])
    # the tile of the stalled block and the later ones of its thread block, no more than all of its tiles
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    width, high, takers = (256, 256, sms // 2) if pairs else (256, 128, sms) if rows > 64 else (128, 16, sms)
    tiles = -(-150000 // width) * -(-rows // high)
    most = -(-tiles // (takers * 3 // 4))  # (a device may hold fewer pairs than half its SMs)
    assert 0 < int(bad.sum()) <= most * width * min(rows, high)
    if block == 0:
        assert bool(bad[0, 0])
    status.zero_()
    assert torch.equal(e3.e3_project_vocab(*ops, status=status), want) and status.item() == 0


def test_refusals(e3):
    x, sx, w, sw = operands(11, 4, 300, 200)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    e3.e3_project_vocab(x, sx, w, sw, status=status)
    assert status.item() == 0
    for bad in ((x.float(), sx, w, sw), (x, sx, w[:, :100], sw), (x, sx[:3], w, sw), (x, sx, w, sw[:2]), (x, sx.double(), w, sw), (x, sx[:, :1], w, sw),
                (x.cpu(), sx, w, sw)):
        with pytest.raises(ValueError):
            e3.e3_project_vocab(*bad)
    for out in (torch.zeros((4, 299), device="cuda"), torch.zeros((4, 300), device="cuda", dtype=torch.float16)):
        with pytest.raises(ValueError):
            e3.e3_project_vocab(x, sx, w, sw, out=out)
    with pytest.raises(e3.E3Error):
        e3.e3_project_vocab(x.contiguous()[:, :200], sx, torch.zeros((300, 200), device="cuda").to(E4M3), sw)  # rows of 200 bytes
    assert e3.e3_project_vocab(x[:0], sx[:0], w, sw).shape == (0, 300)
