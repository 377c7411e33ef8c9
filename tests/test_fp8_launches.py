"""Which kernels the 8-bit products launch, without a GPU: the host half of zs_fp8_gemm.hip with a stand-in for the HIP
runtime (launch_record.cpp) that writes the launches down instead."""
import os
import random
import re
import subprocess

import pytest

from fp8_sizes import PRODUCTS, WORKSPACE
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


TILE = re.compile(r"tiles_kernelILi(\d+)ELi(\d+)ELi(\d+)ELi(\d+)E")


def tile_of(symbol):
    tm, tn, wm, wn = map(int, TILE.search(symbol).groups())
    return 16 * tm * wm, 16 * tn * wn


def splits_of(found, m, n):
    """Into how many parts K is cut."""
    tokens, features = tile_of(found[0][0])
    splits, rest = divmod(found[0][1], -(-m // tokens) * -(-n // features))
    assert rest == 0 and (splits > 1) == (len(found) == 2) and all("join_kernel" in name for name, _ in found[1:])
    return splits


def test_partial_results_fit_the_workspace_and_more_than_128_mb_is_never_used(program):
    rng = random.Random(5)
    sizes = [(rng.randrange(17, 3000), rng.randrange(1, 12000), rng.randrange(1, 15000)) for _ in range(600)]
    rooms = [0, 256, 1 << 20, WORKSPACE, 64 << 20, 128 << 20, 1 << 30]
    found = {room: launches(program, [("f32", *s, 128, room) for s in sizes]) for room in rooms}
    for room in rooms:
        for (m, n, _), f in zip(sizes, found[room]):
            splits = splits_of(f, m, n)
            assert splits == 1 or splits * m * (-(-n // 4) * 4) * 4 <= room
    assert found[128 << 20] == found[1 << 30]
    assert found[0] != found[WORKSPACE] != found[128 << 20]


def test_a_product_that_uses_more_than_the_usual_workspace(program):
    small, large = (launches(program, [("bf16", 473, 8901, 13272, 128, room)])[0] for room in (WORKSPACE, 128 << 20))
    assert splits_of(small, 473, 8901) == 1 and splits_of(large, 473, 8901) > 1


FORMS = [(out, w_rows) for out in ("f32", "bf16") for w_rows in (128, 1)]


@pytest.mark.parametrize("size,tile,split", PRODUCTS)
def test_sizes_of_the_gpu_tests_reach_the_kernels_they_are_meant_for(program, size, tile, split):
    for found in launches(program, [(out, *size[:3], w_rows, size[3]) for out, w_rows in FORMS]):
        if tile is None:
            assert len(found) == 1 and "stream_kernel" in found[0][0]
        else:
            assert tile_of(found[0][0]) == tile and (splits_of(found, *size[:2]) > 1) == split


def test_sizes_of_the_gpu_tests_reach_every_kernel(program):
    every = set(subprocess.run([str(program), "kernels"], capture_output=True, text=True, check=True).stdout.split())
    found = launches(program, [(out, *size[:3], w_rows, size[3]) for size, _, _ in PRODUCTS for out, w_rows in FORMS])
    assert every == {name for f in found for name, _ in f} and len(every) == 18
    unsplit = {f[0][0] for f in found if len(f) == 1}
    split = {f[0][0] for f in found if len(f) == 2}
    assert unsplit == {name for name in every if "join_kernel" not in name}  # results straight to C ...
    assert split == {name for name in every if "tiles_kernel" in name}       # ... and by way of the workspace
