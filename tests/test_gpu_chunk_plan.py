"""How ntp_attn_chunk_shard cuts the walks of row tiles, on a real MI355X: seen in what a call leaves in its workspace.  A piece of a cut walk writes 128 rows of head_dim outputs, a maximum and a
sum; whole walks write none."""
import pytest

from tests.test_gpu_attn_chunk import Case, _say

pytestmark = pytest.mark.gpu
MARK = 0x7fc0beef  # (a NaN that no kernel writes)


def _run(c, parts=0):
    """The call with a workspace of marks: outputs, and how many of the marks are gone."""
    import torch
    N, h = c.N, c.N.ntp_create()
    N.ntp_set_option(N.binding.NTP_OPT_ATTN_PARTS, parts, handle=h)
    need = N.ntp_workspace_bytes(N.binding.NTP_CALL_ATTN_CHUNK_SHARD, c.shape, handle=h)
    ws = torch.full((need // 4,), MARK, dtype=torch.int32, device="cuda")
    N.ntp_set_workspace(ws, handle=h)
    C = torch.full((c.M, c.q * c.d), 77.0, dtype=torch.bfloat16, device="cuda")
    LSE = torch.full((c.q, c.M), 77.0, device="cuda")
    N.ntp_attn_chunk_shard(c.shape, c.pages, c.Q, c.starts_dev, c.table, c.len_dev, C, LSE, handle=h)
    torch.cuda.synchronize()
    N.ntp_destroy(h)
    return C, LSE, int((ws != MARK).sum())


def _pieces(c, written, whole):
    more = written - whole
    assert more % (128 * (c.d + 2)) == 0
    return more // (128 * (c.d + 2))


@pytest.mark.parametrize("fmt,d", [(16, 64), (16, 128), (8, 128)])
@pytest.mark.parametrize("others", [20, 63, 64, 300])
def test_parts_are_those_of_the_option(others, fmt, d):
    """One sequence of two row tiles that walk 63 key tiles, behind `others` of one token each.  A piece has ceil(63 / parts) tiles at most: 32, 13, 5 and 4, of which a walk has 2, 5, 13 and 16."""
    _say(f"parts of one walk behind {others} single tokens, heads of {d}, {fmt} bits")
    c = Case([1] * others + [40], [7 * i % 60 for i in range(others)] + [4000], 4, 1, d, 16, 0, 0, 4, fmt, seed=others)
    C, LSE, whole = _run(c, 1)
    c.check(C, LSE)
    for parts, pieces in ((2, 2), (5, 5), (15, 13), (16, 16)):
        C, LSE, written = _run(c, parts)
        assert _pieces(c, written, whole) == 2 * pieces
        c.check(C, LSE)


@pytest.mark.parametrize("fmt", [16, 8])
@pytest.mark.parametrize("others", [10, 68])
def test_sequences_shorter_than_their_rows_do_not_count_against_the_work(others, fmt):
    """64 tokens behind 31936 (8 row tiles of 500 key tiles), whose walks are worth cutting, beside 2048 rows of a sequence of 5 tokens (256
    row tiles of one): rows that see nothing save no work.  8 * 499.5 + 256 key tiles at most are 8.3 for each of 512 places, and 16.6 for half of them: 30 pieces a walk at least."""
    _say(f"a long walk beside rows that see nothing and {others} single tokens, {fmt} bits")
    c = Case([1] * others + [2048, 64], [i % 50 for i in range(others)] + [5, 32000], 16, 1, 64, 64, 0, 0, 16, fmt, seed=2)
    _, _, whole = _run(c, 1)
    C, LSE, written = _run(c)
    assert _pieces(c, written, whole) >= 8 * 30
    c.check(C, LSE)


@pytest.mark.parametrize("fmt,name", [(16, "attn_chunk"), (8, "attn_chunk8")])
def test_timing_records_name_no_work_that_only_the_device_knows(fmt, name):
    """Bounds far above the lengths: no count of operations that follows from them is the call's."""
    c = Case([3, 50], [30, 100], 4, 1, 64, 16, 0, 0, 4, fmt, max_len=100000, max_new=50)
    N, h = c.N, c.N.ntp_create()
    N.ntp_kernel_timing_enable(True, handle=h)
    C = c.torch.empty(c.M, 256, dtype=c.torch.bfloat16, device="cuda")
    N.ntp_attn_chunk_shard(c.shape, c.pages, c.Q, c.starts_dev, c.table, c.len_dev, C, handle=h)
    records = N.ntp_kernel_timing_read(handle=h)
    N.ntp_destroy(h)
    assert [(r["name"], r["flops"], r["bytes"]) for r in records] == [(name, 0.0, 0.0)] and records[0]["ms"] > 0
