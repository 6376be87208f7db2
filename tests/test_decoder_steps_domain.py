"""Arguments that the steps between the quantised linears turn away at the C entry, without a GPU (made-up pointers, nothing is launched)."""
import pytest

from paper_2608_12932_b200 import binding as B
from paper_2608_12932_b200 import build as libbuild
from tests.test_decoder_steps_abi import cache, vp


@pytest.fixture(scope="module", autouse=True)
def built():
    libbuild.build()


def norm(r, s):
    return B.lib().w4a8_add_rmsnorm_quantize(vp(0x1000), r, vp(0x2000), 1e-6, 4, 256, 128, s, None, vp(0x3000), vp(0x4000), vp(0x5000), None)


def test_norm_does_not_take_a_buffer_that_it_would_leave_unwritten():
    """Without a residual nothing is stored in `sum`: a caller's stream buffer there would keep what it held."""
    assert norm(None, vp(0x8000)) == B.ERR_NULL
    assert norm(vp(0x6000), None) == B.ERR_NULL


@pytest.mark.gpu
def test_the_binding_does_not_either():
    import torch
    x = torch.ones((2, 256), dtype=torch.bfloat16, device="cuda")
    w = torch.ones(256, dtype=torch.bfloat16, device="cuda")
    stream = torch.full_like(x, 7.0)
    with pytest.raises(B.W4A8Error) as e:
        B.w4a8_add_rmsnorm_quantize(x, w, 1e-6, sum_out=stream)
    assert e.value.code == B.ERR_NULL
    torch.cuda.synchronize()
    assert (stream == 7).all()
    assert B.w4a8_add_rmsnorm_quantize(x, w, 1e-6, residual=x, sum_out=stream)[0] is stream
    torch.cuda.synchronize()
    assert (stream == 2).all()


@pytest.mark.parametrize("scale", [float("inf"), float("-inf"), float("nan"), 3.0e38, -3.0e38])
def test_attention_does_not_take_a_scale_that_makes_scores_infinite(scale):
    """In base 2 it is infinite or not a number: rows with nothing but negative products came back as zeros."""
    f = B.lib().w4a8_kv8_attention
    need = B.w4a8_kv8_workspace_bytes(64)

    def code(scale, T=5):
        return f(cache(), vp(0x10000), 384, 3, T, 6, vp(0x30000), 4, vp(0x40000), scale, vp(0x20000), vp(0x50000), need, None)
    assert code(scale) == B.ERR_SHAPE and code(scale, T=0) == B.ERR_SHAPE
    assert code(0.0, T=0) == B.OK and code(-1.0e38, T=0) == B.OK
