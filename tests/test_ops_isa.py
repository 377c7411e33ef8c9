"""Static check of the generated gfx950 code of the 8-bit products and the embedding operators (no GPU): the rules of test_isa_hazards.py,
and the waits of the tiles that go from memory straight to LDS.

tiles_kernel issues its fetches by hand: F of them a block for each wave, STAGES - 1 blocks ahead.  The fetches of a wave complete in
order, so the wait that a block is read behind covers it if the F * (STAGES - 2) fetches of the blocks after it are all that may be
outstanding.  That holds if, on every path, F * (STAGES - 1) vector-memory instructions come before the first such wait and F between one and the
next, and all of them are fetches.  Other waves' fetches have arrived behind the barrier after the wait, and the block that the next fetches
overwrite has been read by all of them if each waited for its LDS reads in front of it."""
import collections
import os
import re
import subprocess

import pytest

from paper_2603_17435_amd import build as zs_build
from test_isa_hazards import VMEM, hazards, kernels, mfma_hazards, successor_function

FETCH = "global_load_lds"


def fetch_faults(ins, fetches, stages):
    """What breaks the rules above: {index: reason}."""
    successors, found = successor_function(ins), {}
    # (fetches since the last wait by hand, is this before the first one, has a barrier followed it)
    seen, work = {0: {(0, True, True)}}, collections.deque([(0, (0, True, True))])
    while work:
        i, (count, first, behind) = work.popleft()
        text, inline = ins[i]
        if not text.endswith(":"):
            mn = text.split()[0]
            if inline and mn == "s_waitcnt" and "vmcnt" in text:
                left = int(re.search(r"vmcnt\((\d+)\)", text).group(1))
                if count != fetches * (stages - 1 if first else 1):
                    found[i] = f"{count} fetches before {text}"
                elif left > fetches * (stages - 2):
                    found[i] = f"{text} leaves a block that is read"
                count, first, behind = 0, False, False
            elif mn == "s_barrier":
                if not (inline and ins[i - 1] == ("s_waitcnt lgkmcnt(0)", True)):
                    found[i] = "barrier without a wait for LDS reads"
                behind = True
            elif mn.startswith(FETCH):
                if not behind:
                    found[i] = "fetch in front of the barrier"
                count += 1
                if count > fetches * (stages - 1 if first else 1):
                    found[i] = "more fetches than the wait allows for"
                    continue
            elif mn.startswith("ds_") and not behind:
                found[i] = "LDS read in front of the barrier"
            elif mn.startswith(VMEM) and count and not first:
                found[i] = f"{text} among the fetches"
        for s in successors(i):
            state = (count, first, behind)
            if s < len(ins) and state not in seen.setdefault(s, set()):
                seen[s].add(state)
                work.append((s, state))
    return found


def test_planted_faults_are_found():
    fetch, wait, reads, barrier = ("global_load_lds_dwordx4 v1, s[4:5]", True), ("s_waitcnt vmcnt(2)", True), ("s_waitcnt lgkmcnt(0)", True), ("s_barrier", True)
    read, label, again, end = ("ds_read_b128 v[4:7], v9", False), (".LBB0_1:", False), ("s_cbranch_scc1 .LBB0_1", False), ("s_endpgm", False)
    everything = ("s_waitcnt vmcnt(0)", True)  # behind the loop
    tail = [again, everything, reads, barrier, end]

    def faults(loop, ahead=4):
        return fetch_faults([fetch] * ahead + [label] + loop + tail, 2, 3)
    assert not faults([wait, reads, barrier, read, fetch, fetch])
    assert faults([wait, reads, barrier, read, fetch])                                            # too few
    assert faults([wait, reads, barrier, read, fetch, fetch, fetch])                              # too many
    assert faults([wait, reads, barrier, read, fetch, fetch], ahead=2)
    assert faults([("s_waitcnt vmcnt(3)", True), reads, barrier, read, fetch, fetch])             # a wait that leaves the block outstanding
    assert faults([wait, reads, read, barrier, fetch, fetch])                                     # read before the others' fetches have arrived
    assert faults([wait, barrier, read, fetch, fetch])                                            # reads of the block before still under way
    assert faults([wait, fetch, reads, barrier, read, fetch])                                     # over a block that others still read
    assert faults([wait, reads, barrier, read, fetch, ("s_cbranch_scc0 .LBB0_2", False), fetch, (".LBB0_2:", False)])  # a path with one fetch
    assert faults([wait, reads, barrier, fetch, ("global_load_dword v3, v[0:1], off", False), fetch])


@pytest.fixture(scope="module")
def asm_of(tmp_path_factory):
    out = tmp_path_factory.mktemp("ops_isa")
    texts = {}
    for src in zs_build.operator_sources():
        to = out / (os.path.basename(src) + ".s")
        cmd = [zs_build.HIPCC, "-S", "--cuda-device-only", src, "-o", str(to)] + \
              [f for f in zs_build.COMMON if f != "-fPIC"] + zs_build.DEVICE
        subprocess.run(cmd, check=True, capture_output=True)
        texts[os.path.basename(src)] = to.read_text()
    return texts


def test_no_hand_written_load_or_matrix_instruction_is_read_too_early(asm_of):
    for source, asm in asm_of.items():
        for name, ins in kernels(asm):
            assert not hazards(ins) and not mfma_hazards(ins), f"{source}: {name}"
            # (fetches to LDS are the only memory access by hand)
            assert all(t.startswith(FETCH) for t, inline in ins if inline and t.startswith(VMEM)), f"{source}: {name}"


def test_tiles_are_read_behind_the_wait_that_covers_them(asm_of):
    seen = 0
    for name, ins in kernels(asm_of["zs_fp8_gemm.hip"]):
        m = re.search(r"tiles_kernelILi(\d+)ELi(\d+)ELi(\d+)ELi(\d+)ELi(\d+)E", name)
        if not m:
            assert not any(t.startswith(FETCH) for t, _ in ins), name
            continue
        seen += 1
        tm, tn, wm, wn, stages = map(int, m.groups())
        fetches = 16 * (tm * wm + tn * wn) // 8 // (wm * wn) + 1
        assert sum(t.startswith(FETCH) for t, _ in ins) >= fetches * stages, name
        found = fetch_faults(ins, fetches, stages)
        assert not found, f"{name}: {list(found.items())[:4]}"
    assert seen == 12
