"""The assembly of the kernel of one new token's attention (no GPU): its LDS reads are inline assembly and its tiles come by DMA, whose order against each other
only the waits in the source keep.  Checked in what the compiler makes of it, along every path."""
import os
import re

import pytest

from paper_2504_06095_amd import build
from tests.test_host_attn_schedule import _code, _in_flight_faults, _symbols, _without_waits


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("asm") / "decode.s")
    build._run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *build.HIP_FLAGS, "-S", "--offload-device-only", "-I", os.path.join(build.ROOT, "include"),
                "-I", build.CSRC, os.path.join(build.CSRC, "ntp_attn_decode.hip"), "-o", out])
    lines = open(out).read().splitlines()
    starts = _symbols(lines, "attn_decode_kernel")
    assert len(starts) == 2  # both head dimensions
    return [_code(lines, s) for s in starts]


def _dma_groups(code):
    """Index of every DMA instruction -> the matrix it brings.  In the text: keys and values before the loop, then the next keys and the next values, eight
    instructions each."""
    at = [i for i, (op, _, text) in enumerate(code) if op.startswith("buffer_load") and re.search(r"\blds\b", text)]
    assert len(at) == 32
    return {i: "KVKV"[n // 8] for n, i in enumerate(at)}


READS = {"ds_read_b128": "K", "ds_read_b64_tr_b16": "V"}


def _tile_faults(code, labels):
    """LDS reads of a tile whose DMA may still be in flight, and DMA into a tile whose reads may be.  State: the matrices of the vector memory instructions
    and of the LDS reads in flight, oldest first; where paths meet, the union, aligned at the youngest."""
    groups = _dma_groups(code)
    state, work, faults = {0: ((), ())}, [0], {}
    merge = lambda a, b: tuple(x | y for x, y in zip((frozenset(),) * (len(b) - len(a)) + a, (frozenset(),) * (len(a) - len(b)) + b))  # noqa: E731
    while work:
        i = work.pop()
        vm, ds = state[i]
        op, _, text = code[i]
        if op == "s_waitcnt":
            for name, q in (("vmcnt", vm), ("lgkmcnt", ds)):
                m = re.search(rf"{name}\((\d+)\)", text)
                if m:
                    q = q[max(len(q) - int(m[1]), 0):]
                if name == "vmcnt":
                    vm = q
                else:
                    ds = q
        elif op.startswith(("buffer_", "global_", "flat_")):
            what = groups.get(i)
            if what and any(what in s for s in ds):
                faults[i] = text
            vm = (*vm, frozenset([what] if what else []))[-70:]
        elif op.startswith(("ds_", "s_load")):
            # (what else is in the LDS lies over the tiles: nothing may be on its way then)
            what = READS.get(op) if op in READS else None
            if op.startswith("ds_") and not op.startswith("ds_bpermute") and any((what in s) if what else s for s in vm):
                faults[i] = text
            ds = (*ds, frozenset([what] if what else []))[-70:]
        after = [] if op == "s_endpgm" else [labels[text.split()[1]]] if op == "s_branch" else [i + 1]
        if op.startswith("s_cbranch"):
            after.append(labels[text.split()[1]])
        for j in after:
            old = state.get(j)
            new = (vm, ds) if old is None else (merge(old[0], vm), merge(old[1], ds))
            if new != old:
                state[j] = new
                work.append(j)
    return faults


def test_tiles_are_read_behind_their_dma_and_overwritten_behind_their_reads(kernels):
    for code, labels in kernels:
        assert not _tile_faults(code, labels)
        # the check sees a wait that leaves more in flight, and one that is missing
        waits = [i for i, (op, _, text) in enumerate(code) if op == "s_waitcnt" and text.endswith("vmcnt(8)")]
        assert len(waits) >= 2
        for w in waits[:2]:
            assert _tile_faults([*code[:w], (code[w][0], code[w][1], "s_waitcnt vmcnt(9)"), *code[w + 1:]], labels)
        assert _tile_faults([c if c[0] != "s_waitcnt" or "lgkmcnt" not in c[2] else ("s_waitcnt", c[1], "s_waitcnt vmcnt(63)") for c in code], labels)


def test_registers_are_left_alone_while_reads_are_in_flight(kernels):
    for code, labels in kernels:
        assert sum(op == "ds_read_b64_tr_b16" for op, _, _ in code) == 32 and not any("scratch_" in text for _, _, text in code)
        assert not _in_flight_faults(code, labels)
        assert _in_flight_faults(_without_waits(code), labels)
