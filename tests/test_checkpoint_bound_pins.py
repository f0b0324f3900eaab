"""The 8-bit checkpoint's scale and its error relative to a block's largest magnitude (CPU, the oracle): the
smallest scale at which the rounded magnitude is at most 127, half a step at most 1/127.5 of it."""
import os
import re

import numpy as np
import pytest

from oracle import operators_oracle as orc

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def below(x, dtype):
    """The next smaller value of the type (bf16: fp32 with 16 bits fewer)."""
    if dtype == "f32":
        return float(np.nextafter(np.float32(x), np.float32(0)))
    return float((np.array([x], np.float32).view(np.uint32) - 0x10000).view(np.float32)[0])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("k", [-120, -7, 0, 3, 119])
def test_scale_around_its_border(dtype, k):
    """127.5 steps go to the next scale, where they are 63.75; what lies below, 127.4 steps too, does not."""
    top = 127.5 * 2.0 ** k
    for x, s, q in ((top, k + 1, 64), (below(top, dtype), k, 127), (127.0 * 2.0 ** k, k, 127), (64.0 * 2.0 ** k, k, 64),
                    (63.75 * 2.0 ** k, k, 64)):
        got_q, got_e = orc.pack(np.array([[x, 0.0]]))
        assert got_e[0, 0] == s + 127 and got_q[0, 0] == q
        # a smaller step would round past 127
        assert np.rint(np.ldexp(x, -(s - 1))) > 127
    q, e = orc.pack(np.array([[127.4, -127.4]]))
    assert e[0, 0] == 127 and q.tolist() == [[127, -127]]


def test_relative_error_of_a_block():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((400, 32)) * np.exp2(rng.uniform(-60, 60, (400, 1)))
    x[:200] *= 127.5 / np.abs(x[:200]).max(1, keepdims=True) * np.exp2(rng.integers(-50, 50, (200, 1)))
    top = np.abs(x).max(1, keepdims=True)
    q, e = orc.pack(x)
    off = np.abs(orc.unpack(q, e) - x)
    assert (off <= top / 127.5 * (1 + 1e-15)).all()
    assert (np.ldexp(0.5, e.astype(int) - 127) <= top / 127.5 * (1 + 1e-15)).all()
    # the bound is met: 127.5 steps of 2^0 and a value a half step of 2 away from a whole one
    x = np.array([[127.5, 1.0]])
    q, e = orc.pack(x)
    assert abs(orc.unpack(q, e)[0, 1] - 1.0) == 127.5 / 127.5
    assert 1 / 127.5 > 2.0 ** -6.995 and 1 / 127.5 > 2.0 ** -7


def test_the_smallest_scale():
    """Below 2^-120 the scale stays at 2^-126, and a value is off by 2^-127 at most."""
    x = np.array([[2.0 ** -127 * 3, 2.0 ** -130]])
    q, e = orc.pack(x)
    assert e[0, 0] == 1 and (np.abs(orc.unpack(q, e) - x) <= 2.0 ** -127).all()


def test_the_header_says_so():
    text = re.sub(r"\s*\n \*\s*", " ", open(os.path.join(ROOT, "include", "flashslice.h")).read())
    assert "smallest >= -126 at which the ROUNDED largest magnitude of the block is at most 127" in text
    assert "1/127.5 = 2^-6.994" in text
    assert "2^-7 of" not in open(os.path.join(ROOT, "paper_2609_32525_gb300", "csrc", "fs_rows.cuh")).read()
