"""ntp_qk_norm_append_shard and ntp_qk_norm_shard_bwd on rows of more heads than a workgroup has threads for (128 of 128 elements, 256 of 64), on a real MI355X: several passes over a token's
heads, the last one with threads left over, with the border between queries and keys inside a pass.  Tolerances as test_gpu_qk_norm.py, whose checks these are (bits in place, alone and again
among them)."""
import pytest

from tests import test_gpu_qk_norm as T

pytestmark = pytest.mark.gpu

WIDE = [
    # M, q, kv, d, rotary, interleaved, pad, gammas
    (5, 96, 96, 128, 128, False, 0, "qk"),
    (600, 96, 96, 128, 128, False, 0, "qk"),   # more tokens than workgroups
    (7, 250, 9, 64, 64, True, 8, "qk"),
    (1100, 250, 9, 64, 32, False, 0, "qk"),
    (33, 100, 31, 128, 64, True, 0, "k"),
    (3, 1, 130, 128, 0, False, 0, "qk"),
]


@pytest.mark.parametrize("fmt", [8, 16])
@pytest.mark.parametrize("M,q,kv,d,rd,inter,pad,gammas", WIDE)
def test_append(M, q, kv, d, rd, inter, pad, gammas, fmt):
    T.test_append(M, q, kv, d, rd, inter, 16, pad, 70000, gammas, fmt)


@pytest.mark.parametrize("workspace", [False, True], ids=["alone", "workspace"])
@pytest.mark.parametrize("M,q,kv,d,rd,inter,pad,gammas", [*WIDE, (9, 300, 0, 64, 64, False, 0, "q")])
def test_gradient(M, q, kv, d, rd, inter, pad, gammas, workspace):
    T.test_gradient(M, q, kv, d, rd, inter, pad, gammas, workspace)
