"""Scalars that the compiler keeps in lanes of vector registers in the kernels of attention over 16-bit rows: read back one by one where they are used,
in the loops too, where a kernel needs more of them than there are.  What a kernel has besides, for the rows in 8 bits, is not to add to them."""
import re
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2504_04704_amd import build

# kernel<type 1, channels, ...>: spilled scalars at most
MOST = {
    "attend_wide_bf16.hip": {"attend_wide_kernel<1, 64, 4": 26, "attend_wide_kernel<1, 128, 4": 59, "attend_wide_kernel<1, 128, 8": 58, "attend_wide_kernel<1, 256, 4": 75},
    "attend_bf16.hip": {"attend_kernel<1, 64, 1, 4, false": 13, "attend_kernel<1, 128, 1, 8, true": 45, "attend_kernel<1, 128, 2, 4, true": 34},
}


def spills(source, tmp):
    out = str(tmp / (source + ".s"))
    subprocess.run([build.hipcc_path(), *build.HIPCC_FLAGS, "-I", build.ROOT + "/include", "-I", build.CSRC, "--cuda-device-only", "-S", build.CSRC + "/" + source,
                    "-o", out], check=True, capture_output=True)
    text = open(out).read()
    names = re.findall(r"\.name:\s+(\S+)\n(?:.*\n)*?\s+\.sgpr_spill_count:\s*(\d+)", text)
    plain = subprocess.run(["c++filt"], input="\n".join(n for n, _ in names), capture_output=True, text=True, check=True).stdout.splitlines()
    return {p: int(n) for p, (_, n) in zip(plain, names)}


@pytest.mark.skipif(subprocess.run(["which", "c++filt"], capture_output=True).returncode != 0, reason="no c++filt")
def test_scalars_kept_in_lanes(tmp_path):
    with ThreadPoolExecutor(2) as ex:
        found = dict(zip(MOST, ex.map(lambda s: spills(s, tmp_path), MOST)))
    for source, most in MOST.items():
        for kernel, n in most.items():
            got = [v for k, v in found[source].items() if kernel in k]
            assert len(got) == 1 and got[0] <= n, (kernel, got, n)
