"""ntp_kv_append_shard against the float64 oracle, on a real MI355X.

Tolerance of a rotated element: half a step of bf16 (2^-8 of the value), and fp32 arithmetic: sine and cosine of an angle known to 2^-24 of half a
turn and within 2 steps of fp32, two products and a sum, 8 * 2^-24 (|x1| + |x2|) together.  What is not rotated is copied bit for bit."""
import sys

import numpy as np
import pytest

from oracle import block_oracle as B

pytestmark = pytest.mark.gpu
U, BF = 2.0 ** -24, 2.0 ** -8


def _say(msg):
    print(f"[gpu-case] {msg}", file=sys.stderr, flush=True)


def f64(t):
    return t.double().cpu().numpy()


def _rand(torch, g, r, c, pad=0):
    full = torch.full((r, c + pad), float("nan"), dtype=torch.bfloat16, device="cuda")
    full[:, :c] = torch.randn(r, c, device="cuda", generator=g)
    return full[:, :c]


def _tol(QKV, want, q, kv, d, rd, inter, first, n):
    """Per element of the heads first .. first + n - 1."""
    M = QKV.shape[0]
    x = np.abs(QKV.reshape(M, q + 2 * kv, d)[:, first:first + n])
    size = np.zeros_like(x)
    if rd:
        a, b = (slice(0, rd, 2), slice(1, rd, 2)) if inter else (slice(0, rd // 2), slice(rd // 2, rd))
        size[..., a] = size[..., b] = x[..., a] + x[..., b]
    size = size.reshape(M, n * d)
    return np.where(size > 0, BF * np.abs(want) + 8 * U * size, 0.0)


CASES = [
    # M, q, kv, d, rotary, interleaved, page, pad, far
    (1, 3, 1, 128, 128, False, 16, 0, 2 ** 31 - 1),
    (64, 3, 1, 128, 128, False, 16, 8, 131072),
    (257, 14, 14, 128, 128, False, 64, 0, 8192),
    (509, 11, 4, 64, 32, True, 32, 40, 1 << 20),
    (33, 7, 2, 64, 64, False, 256, 0, 1000),
    (130, 16, 1, 128, 64, True, 16, 8, 65536),
    (19, 5, 2, 128, 16, False, 128, 0, 100),
    (40, 4, 3, 64, 0, False, 16, 0, 100),
]


@pytest.mark.parametrize("M,q,kv,d,rd,inter,page,pad,far", CASES)
def test_append(M, q, kv, d, rd, inter, page, pad, far):
    import torch
    import paper_2504_06095_amd as N
    _say(f"append {M} tokens, {q} + {kv} heads of {d}, {rd} rotated, pages of {page}")
    g = torch.Generator(device="cuda").manual_seed(M)
    rng = np.random.default_rng(M)
    QKV = _rand(torch, g, M, (q + 2 * kv) * d, pad)
    pos = rng.integers(0, far, M, endpoint=True).astype(np.int32)
    pos[0] = far
    if M > 1:
        pos[1] = 0
    n_pages = (M + page - 1) // page + 2
    slots = rng.permutation(n_pages * page)[:M].astype(np.int64)
    # the padding of a batch, and slots that no page has
    for i, s in ((3, -1), (4, n_pages * page), (5, -(1 << 62)), (6, 1 << 62), (M - 1, -1)):
        if 1 < i < M:
            slots[i] = s
    f = 500000.0 ** (-np.arange(rd // 2) * 2.0 / max(rd, 1))
    # keys and values of a page in one array: pages lie two blocks apart
    both = torch.full((n_pages, 2, kv, page, d), 9.0, dtype=torch.bfloat16, device="cuda")
    K, V = both[:, 0], both[:, 1]
    cache = N.kv_cache(K, V)
    shape = N.kv_append_shape(M, dict(q_cnt=q, kv_cnt=kv, head_dim=d), rd, inter)
    Qout, Kout = _rand(torch, g, M, q * d, pad), _rand(torch, g, M, kv * d, pad)
    dev = (torch.from_numpy(pos).cuda(), torch.from_numpy(slots).cuda(), torch.from_numpy(f).cuda() if rd else None)
    N.ntp_kv_append_shard(shape, cache, QKV, *dev, Qout, Kout)
    torch.cuda.synchronize()
    x = f64(QKV)
    wQ, wKr, wK, wV = B.kv_append(x, q, kv, d, pos, slots, f, inter, np.full((n_pages, kv, page, d), 9.0), np.full((n_pages, kv, page, d), 9.0))
    assert (np.abs(f64(Qout) - wQ) <= _tol(x, wQ, q, kv, d, rd, inter, 0, q)).all()
    assert (np.abs(f64(Kout) - wKr) <= _tol(x, wKr, q, kv, d, rd, inter, q, kv)).all()
    # the cache: exactly Kout's rows and the values in their slots, and nothing else changed
    mark = np.full((n_pages, kv, page, d), 9.0)
    eK, eV, kr = mark.copy(), mark.copy(), f64(Kout).reshape(M, kv, d)
    for m in range(M):
        if 0 <= slots[m] < n_pages * page:
            eK[slots[m] // page, :, slots[m] % page], eV[slots[m] // page, :, slots[m] % page] = kr[m], x.reshape(M, -1, d)[m, q + kv:]
    assert np.array_equal(f64(K), eK) and np.array_equal(f64(V), eV) and np.array_equal(wV, eV)
    if pad:
        assert all(bool(t.as_strided((M, pad), (t.stride(0), 1), t.storage_offset() + t.shape[1]).isnan().all()) for t in (Qout, Kout))
    # in place, the queries alone, the cache alone: the same bits
    P = QKV.clone()
    N.ntp_kv_append_shard(shape, cache, P, *dev, P[:, :q * d], P[:, q * d:(q + kv) * d])
    assert torch.equal(P[:, :q * d], Qout) and torch.equal(P[:, q * d:(q + kv) * d], Kout) and torch.equal(P[:, (q + kv) * d:], QKV[:, (q + kv) * d:])
    Q2 = _rand(torch, g, M, q * d)
    N.ntp_kv_append_shard(shape, None, QKV, dev[0], None, dev[2], Q2, None)
    assert torch.equal(Q2, Qout)
    both.fill_(9.0)
    N.ntp_kv_append_shard(shape, cache, QKV, *dev, None, None)
    torch.cuda.synchronize()
    assert np.array_equal(f64(K), eK) and np.array_equal(f64(V), eV)


def test_no_tokens_and_an_empty_cache():
    import torch
    import paper_2504_06095_amd as N
    e = torch.empty(0, 2, 16, 64, dtype=torch.bfloat16, device="cuda")
    cache = N.kv_cache(e, e)
    f = torch.ones(32, dtype=torch.float64, device="cuda")
    for M in (0, 5):
        QKV = torch.ones(M, 6 * 64, dtype=torch.bfloat16, device="cuda")
        Qout = torch.zeros(M, 2 * 64, dtype=torch.bfloat16, device="cuda")
        N.ntp_kv_append_shard(N.kv_append_shape(M, dict(q_cnt=2, kv_cnt=2, head_dim=64)), cache, QKV, torch.zeros(M, dtype=torch.int32, device="cuda"),
                              torch.zeros(M, dtype=torch.int64, device="cuda"), f, Qout)
        torch.cuda.synchronize()
        assert bool((Qout == 1).all())


def test_slots_behind_four_gigabytes():
    import torch
    import paper_2504_06095_amd as N
    d, page, kv = 128, 65536, 2
    n_pages = 160  # 160 pages of 16.8 M elements: 2.7 G elements, 5.4 GB for K and V each
    K, V = (torch.zeros(n_pages, kv, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    slots = [0, 1, 128 * page - 1, 128 * page, 129 * page + 7, n_pages * page - 1]
    M = len(slots)
    QKV = _rand(torch, torch.Generator(device="cuda").manual_seed(1), M, 6 * d)
    N.ntp_kv_append_shard(N.kv_append_shape(M, dict(q_cnt=2, kv_cnt=2, head_dim=d), 0), N.kv_cache(K, V), QKV, None, torch.tensor(slots, device="cuda"), None)
    torch.cuda.synchronize()
    for m, s in enumerate(slots):
        assert torch.equal(K[s // page, :, s % page].reshape(-1), QKV[m, 2 * d:4 * d]) and torch.equal(V[s // page, :, s % page].reshape(-1), QKV[m, 4 * d:])
    assert int((K != 0).any(3).sum()) == kv * M and int((V != 0).any(3).sum()) == kv * M


# a workgroup takes min(8, 384 / chunk pairs of a row, M / 512) tokens on 256 compute units: 8, 5, 2 and 4 of them here, and a last one with fewer
MANY = [
    (4099, 3, 1, 128, 128, False, 16, 8, 131072),
    (8191, 11, 4, 64, 32, True, 32, 0, 1 << 20),
    (1031, 3, 1, 128, 64, False, 64, 0, 2 ** 31 - 1),
    (2053, 2, 2, 64, 16, True, 256, 40, 4096),
]


@pytest.mark.parametrize("M,q,kv,d,rd,inter,page,pad,far", MANY)
def test_append_of_several_tokens_a_workgroup(M, q, kv, d, rd, inter, page, pad, far):
    test_append(M, q, kv, d, rd, inter, page, pad, far)


def test_outputs_beside_the_columns_of_one_matrix():
    """Queries and keys written into columns of the matrix that holds QKV, which they do not meet: the same bits as elsewhere."""
    import torch
    import paper_2504_06095_amd as N
    M, q, kv, d = 37, 3, 1, 64
    g = torch.Generator(device="cuda").manual_seed(5)
    w = (q + 2 * kv) * d
    wide = _rand(torch, g, M, w + (q + kv) * d)
    f = torch.tensor(10000.0 ** (-np.arange(d // 2) * 2.0 / d), device="cuda")
    pos = torch.arange(M, dtype=torch.int32, device="cuda") * 11
    shape = N.kv_append_shape(M, dict(q_cnt=q, kv_cnt=kv, head_dim=d))
    QKV = wide[:, :w].clone()
    Q, K = (torch.empty(M, n * d, dtype=torch.bfloat16, device="cuda") for n in (q, kv))
    N.ntp_kv_append_shard(shape, None, QKV, pos, None, f, Q, K)
    N.ntp_kv_append_shard(shape, None, wide[:, :w], pos, None, f, wide[:, w:w + q * d], wide[:, w + q * d:])
    torch.cuda.synchronize()
    assert torch.equal(wide[:, :w], QKV) and torch.equal(wide[:, w:w + q * d], Q) and torch.equal(wide[:, w + q * d:], K)


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("d,rd", [(64, 32), (128, 128)])
def test_the_gradient_of_the_rotation_is_the_rotation_back(d, rd, inter):
    """With inv_freq negated, no cache, and the query and key columns of dQKV as outputs.  Against the transposed rotation in float64, and the
    identity sum dY R x = sum (R^T dY) x for what the calls themselves made of x."""
    import torch
    import paper_2504_06095_amd as N
    M, q, kv, far = 213, 5, 2, 100000
    g = torch.Generator(device="cuda").manual_seed(d)
    X, dQKV = _rand(torch, g, M, (q + 2 * kv) * d), _rand(torch, g, M, (q + 2 * kv) * d, 8)
    pos = torch.randint(0, far, (M,), dtype=torch.int32, device="cuda", generator=g)
    f = torch.tensor(500000.0 ** (-np.arange(rd // 2) * 2.0 / rd), device="cuda")
    shape = N.kv_append_shape(M, dict(q_cnt=q, kv_cnt=kv, head_dim=d), rd, inter)
    before, x = f64(dQKV), f64(X)
    wq, wk = q * d, kv * d
    N.ntp_kv_append_shard(shape, None, dQKV, pos, None, -f, dQKV[:, :wq], dQKV[:, wq:wq + wk])
    N.ntp_kv_append_shard(shape, None, X, pos, None, f, X[:, :wq], X[:, wq:wq + wk])
    torch.cuda.synchronize()
    want = before.copy()
    turned = before.reshape(M, -1, d)[:, :q + kv].copy()
    n = rd // 2
    first, second = (slice(0, rd, 2), slice(1, rd, 2)) if inter else (slice(0, n), slice(n, rd))
    a = f64(pos)[:, None, None] * f64(f)
    c, s = np.cos(a), np.sin(a)
    y1, y2 = turned[..., first].copy(), turned[..., second].copy()
    turned[..., first], turned[..., second] = c * y1 + s * y2, c * y2 - s * y1  # transpose of (x1 c - x2 s, x2 c + x1 s)
    want[:, :wq + wk] = turned.reshape(M, -1)
    tol = np.concatenate([_tol(before, want[:, :wq], q, kv, d, rd, inter, 0, q), _tol(before, want[:, wq:wq + wk], q, kv, d, rd, inter, q, kv), np.zeros((M, wk))], 1)
    assert (np.abs(f64(dQKV) - want) <= tol).all()
    # both sides of the identity, row by row: each rounded value is off by half a step of its own, and by 8 fp32 steps of the pair it came from
    rows = slice(0, wq + wk)
    left, right = before[:, rows] * f64(X)[:, rows], f64(dQKV)[:, rows] * x[:, rows]
    slack = np.concatenate([_tol(x, f64(X)[:, :wq], q, kv, d, rd, inter, 0, q), _tol(x, f64(X)[:, wq:wq + wk], q, kv, d, rd, inter, q, kv)], 1)
    # (a half step of the rounded value: (1 + 2^-8) of one of the value itself)
    bound = (1 + BF) * ((np.abs(before[:, rows]) * slack).sum(1) + (tol[:, rows] * np.abs(x[:, rows])).sum(1)) + 1e-9
    assert (np.abs(left.sum(1) - right.sum(1)) <= bound).all()


@pytest.mark.parametrize("q,kv", [(0, 3), (4, 0)])
def test_queries_or_keys_alone(q, kv):
    import torch
    import paper_2504_06095_amd as N
    M, d, page = 45, 64, 16
    X = _rand(torch, torch.Generator(device="cuda").manual_seed(q), M, (q + 2 * kv) * d)
    pos = torch.arange(M, dtype=torch.int32, device="cuda") * 7
    f = torch.tensor(10000.0 ** (-np.arange(d // 2) * 2.0 / d), device="cuda")
    shape = N.kv_append_shape(M, dict(q_cnt=q, kv_cnt=kv, head_dim=d))
    out = torch.zeros(M, (q + kv) * d, dtype=torch.bfloat16, device="cuda")
    K, V = (torch.zeros(3, kv, page, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    if q:
        N.ntp_kv_append_shard(shape, None, X, pos, None, f, out)
    else:
        N.ntp_kv_append_shard(shape, N.kv_cache(K, V), X, pos, torch.arange(M, device="cuda"), f, None, out)
    torch.cuda.synchronize()
    x = f64(X)
    want = B.rotate(x.reshape(M, -1, d)[:, :q + kv], f64(pos), f64(f), False).reshape(M, -1)
    assert (np.abs(f64(out) - want) <= _tol(x, want, q, kv, d, d, False, 0, q + kv)).all()
    if kv:
        rows = lambda t: t.transpose(1, 2).reshape(3 * page, kv * d)[:M]  # noqa: E731
        assert torch.equal(rows(K), out) and torch.equal(rows(V), X[:, kv * d:])
