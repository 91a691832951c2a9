"""Sizes that the 8-bit projection refuses on the host: every one is rejected before a device call."""
import pytest


@pytest.fixture(scope="module")
def e3():
    from paper_2505_18573_b200 import build, binding
    build.build()
    binding.lib()
    return binding


P, MOST = 1 << 20, (1 << 31) - 256  # an aligned address that nothing reads; sizes lie below MOST


@pytest.mark.parametrize("size", [MOST, MOST + 1, MOST + 100, MOST + 127, MOST + 128, MOST + 255, MOST + 256, 1 << 40])
@pytest.mark.parametrize("which", ["rows", "V", "D"])
def test_sizes_from_the_documented_limit_on_are_refused(e3, which, size):
    a = dict(x=P, x_scale=P, rows=3, x_stride=208, x_scale_stride=2, w=P, w_scale=P, V=500, w_stride=208, w_scale_stride=2, D=200, logits=P,
             dt=e3.E3_BF16, row_stride=500, out_status=None, stream=None)
    a[which] = size
    if which == "V":
        a["row_stride"] = size
    if which == "D":
        a["x_stride"] = a["w_stride"] = (size + 15) // 16 * 16
        a["x_scale_stride"] = a["w_scale_stride"] = size // 128 + 1
    assert e3.lib().e3_project_vocab(*a.values()) == e3.E3_ERR_INVALID_ARG
