"""The range of fp16 scales for which the kernels form codes by the reciprocal (quant_common.cuh), on the CPU and step by step in fp32.

The reciprocal form has no clamp: it needs |x / s| < 127.5 - 2^-13.  s is amax / 127 rounded to fp16.  For a normal s the rounding moves the quotient
by a factor of at most 1 + 2^-11.  A subnormal s is n 2^-24 and amax / 127 at most (n + 1/2) 2^-24, so the quotient goes up to 127 (1 + 1 / (2 n)): past
127.5 for n < 127, as far as 190 for n = 1."""
import os
import re

import numpy as np

from oracle import w4a8_oracle as onp

COMMON = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_12932_b200", "csrc", "quant_common.cuh")


def source(name):
    with open(os.path.join(os.path.dirname(COMMON), name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def rule():
    """First scale that takes the reciprocal form, and first that does not any more."""
    m = re.search(r"FAST_SCALE_FIRST = (0x[0-9A-F]+)u, FAST_SCALE_END = (0x[0-9A-F]+)u;", source("quant_common.cuh"))
    return int(m.group(1), 16), int(m.group(2), 16)


def every_bf16():
    return onp.bf16_bits_to_f64(np.arange(0x0001, 0x7F80, dtype=np.uint16))


def scale_bits(amax):
    return np.minimum(amax.astype(np.float32) / np.float32(127.0), np.float32(65504.0)).astype(np.float16).view(np.uint16)


def codes_by_reciprocal(x, s):
    """The low byte of x (1 / s) + 1.5 2^23, and the division with its clamp where the product is near a half-integer."""
    magic, s32, x32 = np.float32(12582912.0), np.float32(s), x.astype(np.float32)
    t = x32 * (np.float32(1.0) / s32)
    y = t + magic
    code = (y.view(np.uint32) & 0xFF).astype(np.uint8).view(np.int8).astype(np.int64)
    near = np.abs(t - (y - magic)) > np.float32(0.5 - 2.0 ** -13)
    return np.where(near, np.clip(np.rint(x32 / s32), -127, 127).astype(np.int64), code)


def test_every_row_whose_scale_is_subnormal():
    """Every bf16 value up to the largest maximum that has this scale, both signs, for every subnormal scale in the rule and the first normal ones."""
    first, end = rule()
    x = every_bf16()
    sb = scale_bits(x)
    assert 1 <= first <= 0x0400 and end == 0x7BFF
    for b in [b for b in np.unique(sb) if first <= b <= 0x0480]:
        s = float(onp.fp16_bits_to_f64(np.array([b], dtype=np.uint16))[0])
        v = x[x <= x[sb == b].max()]
        v = np.concatenate([v, -v])
        want = np.clip(np.rint(v / s), -127, 127).astype(np.int64)
        assert np.array_equal(codes_by_reciprocal(v, s), want), hex(int(b))


def test_every_maximum_has_the_code_127_or_its_definition():
    """The largest magnitude of a row, which is what may pass 127.5, for every scale of the rule."""
    first, end = rule()
    x = every_bf16()
    sb = scale_bits(x)
    wrong_below = 0
    for v, b in zip(x, sb):
        if b == 0 or b >= end:
            continue
        s = float(onp.fp16_bits_to_f64(np.array([b], dtype=np.uint16))[0])
        got = codes_by_reciprocal(np.array([v, -v]), s)
        want = np.clip(np.rint(np.array([v, -v]) / s), -127, 127).astype(np.int64)
        if b >= first:
            assert np.array_equal(got, want), hex(int(b))
        else:
            wrong_below += int(not np.array_equal(got, want))
    assert wrong_below > 0             # what the rule keeps out


def test_every_kernel_asks_the_rule():
    """No kernel that forms codes by the reciprocal has a condition of its own."""
    seen = 0
    for name in sorted(os.listdir(os.path.dirname(COMMON))):
        if not name.endswith(".cu"):
            continue
        text = source(name)
        forms = len(re.findall(r"\.x = quant4_fast\(", text))
        assert forms == len(re.findall(r"fast_scale\(", text)) and not re.search(r"0x7BFF", text), name
        seen += forms
    assert seen == 4
