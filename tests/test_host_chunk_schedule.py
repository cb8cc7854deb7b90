"""The assembly of the kernels of the attention of chunks (no GPU): their LDS reads are inline assembly and tiles come by DMA, whose order against each other only the waits in the
source keep.  Checked in what the compiler makes of it, along every path."""
import os
import re
from itertools import islice

import pytest

from paper_2504_06095_amd import build
from tests import test_host_decode_schedule as D
from tests.test_host_attn_schedule import _code, _in_flight_faults, _symbols, _without_waits


def _in_flight_masks(code, labels):
    """test_host_attn_schedule's check with register sets as bit masks (these kernels have five times its code): the first instructions that touch the destination of an LDS or scalar read
    that may still be in flight."""
    bits = {}
    mask = lambda regs: sum(1 << bits.setdefault(r, len(bits)) for r in regs)  # noqa: E731
    prepared = []
    for op, operands, text in code:
        m = re.search(r"lgkmcnt\((\d+)\)", text) if op == "s_waitcnt" else None
        reads = op.startswith(("ds_", "s_load", "s_buffer_load"))
        after = (labels[text.split()[1]],) if op.startswith(("s_branch", "s_cbranch")) else ()
        prepared.append((op == "s_waitcnt", int(m[1]) if m else None, mask(frozenset().union(*operands)), (mask(operands[0]) if not op.startswith("ds_write") else 0) if reads else None, after,
                         op not in ("s_endpgm", "s_branch")))
    state, work, faults = {0: ()}, [0], {}
    while work:
        i = work.pop()
        q, (wait, left, touched, read, after, falls) = state[i], prepared[i]
        if wait:
            q = q if left is None else q[max(len(q) - left, 0):]
        else:
            if any(touched & x for x in q):
                faults[i] = code[i][2]
            if read is not None:
                q = (*q, read)
        for j in (*after, *((i + 1,) if falls else ())):
            old = state.get(j)
            if old is None:
                new = q
            else:
                n = max(len(old), len(q))
                new = tuple(a | b for a, b in zip((0,) * (n - len(old)) + old, (0,) * (n - len(q)) + q))
            new = new[-32:]
            if new != old:
                state[j] = new
                work.append(j)
    return faults


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    out = str(tmp_path_factory.mktemp("asm") / "chunk.s")
    build._run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *build.HIP_FLAGS, "-S", "--offload-device-only", "-I", os.path.join(build.ROOT, "include"),
                "-I", build.CSRC, os.path.join(build.CSRC, "ntp_attn_chunk.hip"), "-o", out])
    return open(out).read().splitlines()


@pytest.mark.parametrize("kernel,count", [("chunk_rows_kernel", 8), ("chunk_tiles_kernel", 4), ("chunk_both_kernel", 4)])
def test_registers_are_left_alone_while_reads_are_in_flight(assembly, kernel, count):
    starts = _symbols(assembly, kernel)
    assert len(starts) == count
    for start in starts:
        code, labels = _code(assembly, start)
        assert sum("_tr_b" in op for op, _, _ in code) >= 16 and not any("scratch_" in text for _, _, text in code), assembly[start]
        assert not _in_flight_masks(code, labels), assembly[start]
        assert _in_flight_masks(_without_waits(code), labels)
    if kernel == "chunk_tiles_kernel":  # (the same faults as by the plain check)
        assert set(_in_flight_masks(_without_waits(code), labels)) == set(_in_flight_faults(_without_waits(code), labels))


def test_tiles_are_read_behind_their_dma_and_overwritten_behind_their_reads(assembly, monkeypatch):
    """The kernels whose wavefronts have tiles of their own, without barriers between the tiles."""
    monkeypatch.setattr(D, "READS", {"ds_read_b128": "K", "ds_read_b64": "K", "ds_read_b64_tr_b16": "V", "ds_read_b64_tr_b8": "V"})

    def groups(code):
        at = [i for i, (op, _, text) in enumerate(code) if op.startswith("buffer_load") and re.search(r"\blds\b", text)]
        assert len(at) in (16, 32)  # keys and values, before the loop and in it
        return {i: "KVKV"[n * 4 // len(at)] for n, i in enumerate(at)}

    monkeypatch.setattr(D, "_dma_groups", groups)
    for start in _symbols(assembly, "chunk_rows_kernel"):
        code, labels = _code(assembly, start)
        faults = D._tile_faults(code, labels)
        assert not faults, (assembly[start], list(faults.values())[:5])
        n = len(groups(code)) // 4
        waits = [i for i, (op, _, text) in enumerate(code) if op == "s_waitcnt" and text.endswith(f"vmcnt({n})")]
        assert len(waits) >= 2
        late = (i for i in waits if D._tile_faults([*code[:i], (code[i][0], code[i][1], f"s_waitcnt vmcnt({n + 1})"), *code[i + 1:]], labels))
        assert len(list(islice(late, 2))) == 2, assembly[start]  # (the check sees waits that leave more in flight, and missing ones)
        assert D._tile_faults([c if c[0] != "s_waitcnt" or "lgkmcnt" not in c[2] else ("s_waitcnt", c[1], "s_waitcnt vmcnt(63)") for c in code], labels)
