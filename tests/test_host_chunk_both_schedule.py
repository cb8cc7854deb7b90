"""The assembly of the chunk attention kernels that take row tiles (no GPU): the order of what brings a tile into the LDS, the waits, the barriers and the inline assembly's reads, along every
path.  bf16 tiles come by DMA, 8-bit ones by LDS writes from registers; two buffers, which all wavefronts fill and read.  The kernels that hold workgroups of both kinds have a walk of few
rows of their own, with waits by count."""
import re
from itertools import islice

import pytest

from tests import test_host_decode_schedule as D
from tests.test_host_attn_schedule import _code, _symbols
from tests.test_host_chunk_schedule import assembly  # noqa: F401

KERNELS = [(k, d, fp8) for k in ("chunk_tiles_kernel", "chunk_both_kernel") for d in (64, 128) for fp8 in (False, True)]
DMA = re.compile(r"\blds\b")


def _kernel(lines, kernel, d, fp8):
    start, = (i for i in _symbols(lines, kernel) if f"ILi{d}ELb{int(fp8)}E" in lines[i])
    return _code(lines, start)


def _buffers(code, d, fp8, order=(0, 1, 0)):
    """Instruction -> ("bring" | "read", buffer) of the walk over key tiles, which lies behind the choice of the cuts (the last 32-bit LDS writes).  In the text the first tile is brought before the
    loop, the loop's halves bring into the other buffer than they read; the reads' offsets name theirs."""
    first = 1 + max(i for i, (op, _, _) in enumerate(code) if re.fullmatch(r"ds_write2?_b32", op))
    brings = [i for i in range(first, len(code)) if (code[i][0] == "ds_write_b128" if fp8 else code[i][0].startswith("buffer_load") and DMA.search(code[i][2]))]
    assert len(brings) == 3 * d // 16
    what = {i: ("bring", order[n * 3 // len(brings)]) for n, i in enumerate(brings)}
    reads = [i for i in range(brings[0], len(code)) if code[i][0] in ("ds_read_b128", "ds_read_b64_tr_b16")]
    of = lambda i: int((re.search(r"offset:(\w+)", code[i][2]) or [0, "0"])[1], 0) // (64 * d * 2)  # noqa: E731
    last = max(i for i in reads if code[i][0] == "ds_read_b64_tr_b16")
    what.update({i: ("read", of(i)) for i in reads if i <= last})
    assert sum(w == ("read", 0) for w in what.values()) == sum(w == ("read", 1) for w in what.values()) >= 24
    return what


def _buffer_faults(code, labels, what, fp8):
    """Reads of a buffer that some wavefront's share may not have reached, and shares brought into one that some wavefront may still read.  Per buffer, over all paths: "sent" (brought, not waited
    for), "here" (waited for, no barrier since), "read" (since the last barrier), "reading" (not waited for)."""
    clean = (frozenset(), frozenset())
    state, work, faults = {0: clean}, [0], {}
    while work:
        i = work.pop()
        s, (op, _, text) = [set(x) for x in state[i]], code[i]
        if op == "s_waitcnt":
            for x in s:
                if re.search(r"lgkmcnt\(0\)" if fp8 else r"vmcnt\(0\)", text) and "sent" in x:
                    x.discard("sent"), x.add("here")
                if "lgkmcnt(0)" in text:
                    x.discard("reading")
        elif op == "s_barrier":
            for x in s:
                x.discard("here")
                if "reading" not in x:
                    x.discard("read")
        elif i in what:
            kind, b = what[i]
            if s[b] & ({"read", "reading"} if kind == "bring" else {"sent", "here"}):
                faults[i] = text
            s[b] |= {"sent"} if kind == "bring" else {"read", "reading"}
        after = [] if op == "s_endpgm" else [labels[text.split()[1]]] if op == "s_branch" else [i + 1]
        if op.startswith("s_cbranch"):
            after.append(labels[text.split()[1]])
        for j in after:
            new = tuple(frozenset(a) | b for a, b in zip(s, state.get(j, clean)))
            if j not in state or new != state[j]:
                state[j] = new
                work.append(j)
    return faults


@pytest.mark.parametrize("kernel,d,fp8", KERNELS)
def test_tiles_of_all_wavefronts_are_there_before_they_are_read(assembly, kernel, d, fp8):  # noqa: F811
    code, labels = _kernel(assembly, kernel, d, fp8)
    what = _buffers(code, d, fp8)
    assert not _buffer_faults(code, labels, what, fp8)
    # the check sees a missing barrier, missing waits (of what is brought, and of reads), and shares that go into the wrong buffer
    first, last = min(what), max(what)
    barriers = [i for i in range(first, last) if code[i][0] == "s_barrier"]
    assert len(barriers) == 2
    without = lambda gone: [("s_nop", c[1], "s_nop 0") if gone(i, c) else c for i, c in enumerate(code)]  # noqa: E731
    for b in barriers:
        assert _buffer_faults(without(lambda i, c: i == b), labels, what, fp8)
    for count in ("lgkmcnt(0)",) if fp8 else ("vmcnt(0)", "lgkmcnt(0)"):
        assert _buffer_faults(without(lambda i, c: c[0] == "s_waitcnt" and count in c[2]), labels, what, fp8), count
    assert _buffer_faults(code, labels, _buffers(code, d, fp8, (1, 0, 1)), fp8)


@pytest.mark.parametrize("d,fp8", [(d, fp8) for d in (64, 128) for fp8 in (False, True)])
def test_few_rows_beside_row_tiles(assembly, monkeypatch, d, fp8):  # noqa: F811
    """test_host_chunk_schedule's check of the walk of few rows, in the kernels that hold both: its DMA passes the caches (nt), that of row tiles does not."""
    monkeypatch.setattr(D, "READS", {"ds_read_b128": "K", "ds_read_b64": "K", "ds_read_b64_tr_b16": "V", "ds_read_b64_tr_b8": "V"})

    def groups(code):
        at = [i for i, (op, _, text) in enumerate(code) if op.startswith("buffer_load") and DMA.search(text) and re.search(r"\bnt\b", text)]
        assert len(at) == (16 if fp8 else 32)  # keys and values, before the loop and in it
        return {i: "KVKV"[n * 4 // len(at)] for n, i in enumerate(at)}

    monkeypatch.setattr(D, "_dma_groups", groups)
    code, labels = _kernel(assembly, "chunk_both_kernel", d, fp8)
    faults = D._tile_faults(code, labels)
    assert not faults, list(faults.values())[:5]
    n, end = len(groups(code)) // 4, max(groups(code))
    waits = [i for i, (op, _, text) in enumerate(code[:end]) if op == "s_waitcnt" and text.endswith(f"vmcnt({n})")]
    late = (i for i in waits if D._tile_faults([*code[:i], (code[i][0], code[i][1], f"s_waitcnt vmcnt({n + 1})"), *code[i + 1:]], labels))
    assert len(list(islice(late, 2))) == 2  # (the check sees waits that leave more in flight, and missing ones)
    assert D._tile_faults([c if c[0] != "s_waitcnt" or "lgkmcnt" not in c[2] else ("s_waitcnt", c[1], "s_waitcnt vmcnt(63)") for c in code], labels)
