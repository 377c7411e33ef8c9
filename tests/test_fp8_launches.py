"""Which kernels the 8-bit products launch, without a GPU: the host half of zs_fp8_gemm.hip with a stand-in for the HIP
runtime (launch_record.cpp) that writes the launches down instead."""
import os
import re
import subprocess

import pytest

from fp8_sizes import WORKSPACE
from paper_2603_17435_amd import build as zs_build

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    out = tmp_path_factory.mktemp("launches")
    host, record, exe = out / "host.o", out / "record.o", out / "program"
    common = list(zs_build.COMMON)

    def run(cmd):
        return subprocess.run([str(c) for c in cmd], check=True, capture_output=True, text=True).stdout
    run([zs_build.HIPCC, "-c", "--cuda-host-only", "--offload-arch=gfx950", "-Wno-int-to-pointer-cast", os.path.join(zs_build.OPS, "zs_fp8_gemm.hip"),
         "-o", host] + common)
    run([zs_build.HIPCC, "-x", "c++", "-c", os.path.join(HERE, "launch_record.cpp"), "-o", record, "-D__HIP_PLATFORM_AMD__",
         "-I", "/opt/rocm/include"] + common)
    # the kernels' code, which is not there and not needed
    device_code = [w.split()[-1] for w in run(["nm", host]).splitlines() if re.search(r"__hip_fatbin_[0-9a-f]", w)]
    run(["g++", "-o", exe, host, record] + [f"-Wl,--defsym={s}=0" for s in device_code])
    return exe


def launches(program, products):
    """For each ("f32" or "bf16", M, N, K, w_rows, bytes of workspace): [(kernel's symbol, workgroups)]."""
    text = "".join(" ".join(map(str, p)) + "\n" for p in products)
    done = subprocess.run([str(program)], input=text, capture_output=True, text=True, timeout=60, check=True).stdout.splitlines()
    found = []
    for line in done:
        status, *rest = line.split()
        assert status == "0", line
        found.append(list(zip(rest[::2], map(int, rest[1::2]))))
    assert len(found) == len(products)
    return found


@pytest.mark.parametrize("out,m,n,k,few", [("f32", 1, 28672, 8192, True),     # 44 us against 54 in tiles
                                           ("f32", 16, 28672, 4096, True),    # 28.1 against 30.8
                                           ("f32", 7, 32768, 1024, False),    # 13.3 against 10.5
                                           ("bf16", 11, 32768, 1024, False),  # 13.6 against 10.0
                                           ("bf16", 16, 4096, 4096, True)])   # 8.4 against 11.4
def test_few_tokens_take_the_kernel_that_measured_faster(program, out, m, n, k, few):
    (first, *_), = launches(program, [(out, m, n, k, 128, WORKSPACE)])
    assert ("stream_kernel" in first[0]) == few, first
