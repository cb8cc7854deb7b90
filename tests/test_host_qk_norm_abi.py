"""Gradients of the norms' weights in the same memory: refused, since the two are written side by side (one gamma for queries and keys has two gradients, which the caller adds)."""
from tests.test_host_block_abi import P, _has_gpu, h  # noqa: F401
from tests.test_host_chunk_abi import INV, NODEV, _bwd


def test_gradients_of_the_gammas_share_nothing(h):  # noqa: F811
    for db in (9 * P, 9 * P + 4, 9 * P + 252, 9 * P - 252):
        assert _bwd(h, da=9 * P, db=db) == INV, db
        assert _bwd(h, dict(M=0), da=9 * P, db=db) == INV, db
    assert _bwd(h, dict(head_dim=128), da=9 * P, db=9 * P + 508, ldqkv=640, lddq=384, lddk=128, lddqkv=640) == INV
    if not _has_gpu():  # (with one, the calls would run)
        for db in (9 * P + 256, 9 * P - 256, None):
            assert _bwd(h, da=9 * P, db=db) == NODEV, db
        assert _bwd(h, da=None, db=9 * P) == NODEV
