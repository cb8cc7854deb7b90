"""Which kernels of the block norms the tables of test_gpu_norm_paths.py reach (no GPU): the host's rules for 256 compute units, written out again."""
from tests.test_gpu_norm_paths import BACKWARD, FORWARD

CHUNK, MOST = 8, 4  # columns of a chunk, chunks of a thread


def _threads(H):
    t = 64
    while CHUNK * MOST * t < H:
        t *= 2
    return t


def _chunks(H, t):
    return -(-(H // CHUNK) // t)


def _forward(M, H):
    t = _threads(H)
    while _chunks(H, t) > 1 and 2 * t <= 1024 and M * t * 2 <= 256 * 1024:
        t *= 2
    return _chunks(H, t)


def _backward(H):
    t = _threads(H)
    if _chunks(H, t) == MOST and 2 * t <= 512:
        t *= 2
    return "long" if t > 512 else _chunks(H, t)


def test_every_forward_kernel_runs():
    assert {(_forward(M, H), fp32) for M, H, *_, fp32, _, _, _ in FORWARD} == {(v, f) for v in (1, 2, 3, 4) for f in (False, True)}


def test_every_backward_kernel_runs():
    assert {(_backward(H), kind, fp32) for _, H, kind, fp32 in BACKWARD} == {(v, k, f) for v in (1, 2, 3, 4, "long") for k in range(4) for f in (False, True)}
