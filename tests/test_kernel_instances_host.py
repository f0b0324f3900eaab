"""Every compiled kernel of the layer norm's backward is one that some call reaches, and every one that a
call reaches is there: the rule that chooses them, over all widths, against the library's symbols."""
import re
import shutil
import subprocess

import pytest

from test_abi_host import LIB, fs  # noqa: F401  (builds the library if it is not there)

SIZE = {"f": 4, "13__nv_bfloat16": 2}


# channels of a vector: most vectors of a row, its threads, vectors of a thread
LANES = {8: [(8, 8, 1), (32, 32, 1), (64, 32, 2), (128, 128, 1), (256, 128, 2), (512, 512, 1), (1024, 512, 2)],
         4: [(8, 8, 1), (32, 32, 1), (64, 32, 2), (128, 32, 4), (256, 128, 2), (512, 128, 4), (1024, 512, 2), (2048, 512, 4)],
         2: [(32, 32, 1), (64, 32, 2), (128, 32, 4), (256, 32, 8), (512, 128, 4), (1024, 128, 8), (2048, 512, 4), (4096, 512, 8)],
         1: [(32, 32, 1), (64, 32, 2), (128, 32, 4), (256, 32, 8), (512, 128, 4), (1024, 128, 8), (4096, 512, 8), (8192, 512, 16)]}


def lanes(C, size):
    ve = next(v for v in (8, 4, 2, 1) if v <= 16 // size and C % v == 0)
    return (ve, *next(row[1:] for row in LANES[ve] if -(-C // ve) <= row[0]))


def kernels(C, size, res, ckpt, many):
    ve, threads, k = lanes(C, size)
    n = ve * k
    if threads == 32:
        nd = 16 * C * size
        stage = nd * (2 if res else 1) + (16 * (C + -(-C // 32)) if ckpt else nd)
        for per_sm in (3, 2) if n <= 8 else (2,):
            fit = (232448 // per_sm - 2048) // stage
            if fit >= 2:
                if n > 8 or ve == 1 or (ve == 8 and fit >= 3 and many):
                    return ("15k_norm_bwd_bulk", ve, k, int(ckpt), int(ckpt and ve == 8 and C == 32 * n))
                break
    return ("10k_norm_bwd", ve, threads, k, int(ckpt))


@pytest.mark.skipif(not shutil.which("nm"), reason="lists the library's symbols")
def test_the_backwards_kernels_are_those_that_calls_reach(fs):
    names = subprocess.run(["nm", LIB], capture_output=True, text=True, check=True).stdout
    built = set()
    for kernel, dtype, args in re.findall(r"_ZN2fs4rows(15k_norm_bwd_bulk|10k_norm_bwd)I(f|13__nv_bfloat16)((?:L[ib]\d+E)+)EEvNS", names):
        built.add((dtype, kernel, *map(int, re.findall(r"L[ib](\d+)E", args))))
    reached = {(dtype, *kernels(C, size, res, ckpt, many)) for dtype, size in SIZE.items() for C in range(1, 8193)
               for res in (False, True) for ckpt in (False, True) for many in (False, True)}
    assert built - reached == set()   # compiled, and never launched
    assert reached - built == set()
