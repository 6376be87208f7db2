"""The status word that the 8-bit cache's kernels share with the linears: what says that an output is invalid is not lost to what says that a position
was left out."""
import numpy as np
import pytest
import torch

from paper_2608_12932_b200 import binding as B
from tests.test_gpu_decoder_steps import attend_case, causal, i32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T", [1, 8, 150])
def test_an_earlier_timeout_stays(T):
    """The word as a bounded wait leaves it (written from the host), then calls that meet a block number and a start that do not exist."""
    _, c, table, q = attend_case(T + 80, 1, T, 2, 4, 64, 16, 200)
    word = c.ws[:4].view(torch.int32)
    table[0, 1] = -1
    k = torch.ones((T, 2, 64), dtype=torch.bfloat16, device="cuda")
    calls = [lambda: c.attend(q, table, causal([200], T), 0.1),
             lambda: B.w4a8_kv8_append(c.dev, k, k, i32(table), i32([17]), c.ws),
             lambda: B.w4a8_kv8_append(c.dev, k, k, i32(table), i32([-1]), c.ws)]
    for call in calls:
        for earlier, want in ((B.ERR_TIMEOUT, B.ERR_TIMEOUT), (0, B.ERR_INDEX), (B.ERR_INDEX, B.ERR_INDEX)):
            word.fill_(earlier)
            call()
            with pytest.raises(B.W4A8Error) as e:
                B.w4a8_check_status(c.ws)
            assert e.value.code == want
            B.w4a8_check_status(c.ws)                         # cleared
