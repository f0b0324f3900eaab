"""The shared memory that a kernel may be launched with is a property of the function, which all
host threads share: it is set to one constant per kernel, never to what one call needs."""
import glob
import os
import re

SRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_32525_gb300", "csrc")


def sources():
    return {os.path.basename(f): open(f).read() for f in glob.glob(os.path.join(SRC, "*.cu*")) + glob.glob(os.path.join(SRC, "*.h"))}


def test_only_one_place_sets_a_kernels_limit():
    assert [n for n, s in sources().items() if "cudaFuncSetAttribute" in s] == ["fs_launch.h"]
    body = re.search(r"template <size_t kBytes, typename Kernel>\ncudaError_t allow_smem\(Kernel kernel\) \{(.*?)\}",
                     sources()["fs_launch.h"], re.S).group(1)
    assert "(int)kBytes" in body


def test_every_use_gives_a_constant():
    # a template argument is a constant; the kernel is the only argument at run time
    uses = [line for n, s in sources().items() if n != "fs_launch.h" for line in s.splitlines() if "allow_smem" in line]
    assert len(uses) >= 14 and all(re.search(r"\ballow_smem<.+>\(k\w*\)", line) for line in uses)
