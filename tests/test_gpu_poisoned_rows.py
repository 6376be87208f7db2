"""A row of q with an infinity or not-a-number gives not-a-number in that row alone, whatever the signs of its products, and zeros where it sees no key."""
import numpy as np
import pytest
import torch

from tests.test_gpu_decoder_steps import attend_case, causal

pytestmark = pytest.mark.gpu

INF, NAN = 0x7F80, 0x7FC0
VALUES = (INF, INF | 0x8000, NAN, NAN | 0x8000, 0x7F81)


def check(c, q, table, limits, poison, where, channel, empty=()):
    """`where`: poisoned (sequence, token, head) places; those in `empty` see no key."""
    B_, T, heads, dim = q.shape
    clean = c.attend(q, table, limits, 0.1).view(B_, T, heads, dim).clone()
    bad = q.copy()
    for place in where:
        bad[place][channel] = poison
    got = c.attend(bad, table, limits, 0.1).view(B_, T, heads, dim)
    for place in where:
        if place in empty:
            assert (got[place] == 0).all()
        else:
            assert torch.isnan(got[place]).all()
        got[place] = clean[place]
    assert torch.equal(got, clean)


@pytest.mark.parametrize("T", [1, 8, 150])
@pytest.mark.parametrize("dim,sign", [(64, 1), (64, -1), (128, 1), (128, -1)])
def test_the_first_token_of_a_prompt(T, dim, sign):
    """One visible key: every score of the row has one sign."""
    _, c, table, q = attend_case(T + dim, 1, T, 2, 4, dim, 16, T)
    c.k[table[0, 0], :, 0, 17] = 5 * sign
    c.upload()
    for poison in VALUES:
        check(c, q, table, causal([T], T), poison, [(0, 0, 5), (0, 0, 2)], 17)


@pytest.mark.parametrize("T", [1, 8, 150])
@pytest.mark.parametrize("code", [-50, 0, 50])
def test_products_of_one_sign_over_many_keys(T, code):
    """All keys push the score the same way, or not at all, over several slices of the keys."""
    _, c, table, q = attend_case(T + 70, 2, T, 2, 4, 128, 32, 1700)
    c.k[..., 100] = code
    c.upload()
    limits = causal([1700, 900], T)
    for poison in VALUES:
        check(c, q, table, limits, poison, [(0, T - 1, 3), (1, T // 2, 0)], 100)


@pytest.mark.parametrize("T", [1, 8, 150])
def test_scales_of_zero(T):
    """Infinity times nothing is not a number either: keys of scale zero, then values."""
    _, c, table, q = attend_case(T + 71, 1, T, 2, 4, 64, 16, 200)
    c.ks[:] = 0
    c.upload()
    for poison in VALUES:
        check(c, q, table, causal([200], T), poison, [(0, T // 2, 6)], 1)
    c.vs[:], c.v[:] = 0, 0
    c.upload()
    check(c, q, table, causal([200], T), INF, [(0, T // 2, 6)], 1)


@pytest.mark.parametrize("T", [1, 8, 150])
def test_rows_without_a_key(T):
    """No position visible, or only such whose block does not exist."""
    _, c, table, q = attend_case(T + 72, 3, T, 2, 4, 128, 16, 300)
    limits = causal([300, 300, 300], T)
    limits[0, T // 2] = 0
    table[1] = -1                                             # the whole sequence
    table[2, 2:] = c.k.shape[0]                               # all but 32 positions
    for poison in VALUES:
        check(c, q, table, limits, poison, [(0, T // 2, 1), (1, T - 1, 7), (2, T - 1, 4)], 64, empty=((0, T // 2, 1), (1, T - 1, 7)))


@pytest.mark.parametrize("T", [1, 8, 150])
def test_every_row(T):
    _, c, table, q = attend_case(T + 73, 2, T, 1, 4, 64, 64, 130)
    limits = causal([130, 40], T)
    got = c.attend(np.full_like(q, NAN), table, limits, 0.1).view(2, T, -1)
    seen = torch.from_numpy(limits > 0).cuda()
    assert torch.isnan(got[seen]).all() and (got[~seen] == 0).all()
