"""ntp_qk_norm_append_shard and ntp_qk_norm_shard_bwd against the float64 oracle, on a real MI355X.

Tolerances, U = 2^-24 (half a step of fp32): a head's sum of squares (at most 128 positive terms, 16 in a row and 3 exchanges) has an error of at most 20 U of itself, its
reciprocal root half of that and 2 U; a normed element y = x rstd gamma 14 U |y|.  The rotation adds what the append's tests count, 8 U (|y1| + |y2|): together 24 U (|y1|
+ |y2|).  bf16 outputs: half a step of 2^-8 of the value besides.  e4m3: half a step, 2^-4 of the value, or in the type's lowest range 2^-10 of the head's power of two.
Gradient: with u the gradient turned back (8 U (|u1| + |u2|)) and w = u gamma, the product w . xh is a sum of at most 128 terms with 40 U of the sum of their sizes S; dx = rstd (w -
xh S / d) then has an error of at most 64 U rstd (|w1| + |w2| sizes + |xh| S / d), and half a step of bf16.  A gamma's gradient is a sum over n = tokens x heads terms, each
with at most 40 U, in partial sums of at most 4096 in a row: 1e-5 of the sum of their sizes bounds all of it for n up to 10^6 (random signs of the additions' errors; the worst case of
4096 U = 2.4e-4 is not met by fp32 sums of terms of either sign)."""
import sys

import numpy as np
import pytest

from oracle import block_oracle as B

pytestmark = pytest.mark.gpu
U, BF, EPS = 2.0 ** -24, 2.0 ** -8, 1e-6


def _say(msg):
    print(f"[gpu-case] {msg}", file=sys.stderr, flush=True)


def f64(t):
    return t.float().double().cpu().numpy()


def _rand(torch, g, r, c, pad=0, std=1.0):
    full = torch.full((r, c + pad), float("nan"), dtype=torch.bfloat16, device="cuda")
    full[:, :c] = torch.randn(r, c, device="cuda", generator=g) * std
    return full[:, :c]


def _pairs(size, rd, inter):
    """|y1| + |y2| of the pair that an element is turned in, or |y|."""
    size = size.copy()
    if rd:
        a, b = (slice(0, rd, 2), slice(1, rd, 2)) if inter else (slice(0, rd // 2), slice(rd // 2, rd))
        size[..., a] = size[..., b] = size[..., a] + size[..., b]
    return size


class Case:
    def __init__(self, M, q, kv, d, rd, inter, page, pad, far, gammas="qk", fmt=8, seed=0):
        import torch
        import paper_2504_06095_amd as N
        self.torch, self.N, self.M, self.q, self.kv, self.d, self.rd, self.inter, self.page, self.pad, self.fmt = torch, N, M, q, kv, d, rd, inter, page, pad, fmt
        g = self.g = torch.Generator(device="cuda").manual_seed(M + seed)
        rng = np.random.default_rng(M + seed)
        self.QKV = _rand(torch, g, M, (q + 2 * kv) * d, pad, 3.0)
        if M > 2:  # heads of very different sizes, and one of zeros
            self.QKV[1] *= 2.0 ** -30
            self.QKV[2, :] = 0
        self.gq = (1 + 0.3 * torch.randn(d, device="cuda", generator=g)).bfloat16() if "q" in gammas else None
        self.gk = (1 + 0.3 * torch.randn(d, device="cuda", generator=g)).bfloat16() if "k" in gammas else None
        self.norm = N.qk_norm(self.gq, self.gk, EPS) if gammas else None
        pos = rng.integers(0, far, M, endpoint=True).astype(np.int32)
        pos[0] = far
        self.pos = pos
        self.n_pages = (M + page - 1) // page + 2
        slots = rng.permutation(self.n_pages * page)[:M].astype(np.int64)
        for i, s in ((3, -1), (4, self.n_pages * page), (5, -(1 << 62)), (6, 1 << 62), (M - 1, -1)):
            if 1 < i < M:
                slots[i] = s
        self.slots = slots
        self.f = 500000.0 ** (-np.arange(rd // 2) * 2.0 / max(rd, 1))
        self.dev = (torch.from_numpy(pos).cuda(), torch.from_numpy(slots).cuda(), torch.from_numpy(self.f).cuda() if rd else None)
        self.shape = N.kv_append_shape(M, dict(q_cnt=q, kv_cnt=kv, head_dim=d), rd, inter)
        self.fresh()

    def fresh(self):
        """Pages (keys and values in one array: pages lie two blocks apart) full of a mark."""
        torch, n, kv, page, d = self.torch, self.n_pages, self.kv, self.page, self.d
        if self.fmt == 8:
            self.both = torch.full((n, 2, kv, page, d), 0x33, dtype=torch.uint8, device="cuda")
            self.exps = torch.full((n, 2, kv, page), 99, dtype=torch.uint8, device="cuda")
            self.pages = self.N.kv_pages(self.both[:, 0].view(torch.float8_e4m3fn), self.both[:, 1].view(torch.float8_e4m3fn), self.exps[:, 0], self.exps[:, 1].view(torch.float8_e8m0fnu))
        else:
            self.both = torch.full((n, 2, kv, page, d), 9.0, dtype=torch.bfloat16, device="cuda")
            self.exps = None
            self.pages = self.N.kv_pages(self.both[:, 0], self.both[:, 1])

    def exact(self):
        o = lambda t: None if t is None else f64(t)  # noqa: E731
        return B.qk_norm(f64(self.QKV), self.q, self.kv, self.d, o(self.gq), o(self.gk), EPS, self.pos, self.f, self.inter)

    def sizes(self):
        x = f64(self.QKV).reshape(self.M, -1, self.d)
        o = lambda t: None if t is None else f64(t)  # noqa: E731
        y = [np.abs(B.head_norm(x[:, :self.q], o(self.gq), EPS)), np.abs(B.head_norm(x[:, self.q:self.q + self.kv], o(self.gk), EPS))]
        return [_pairs(t, self.rd, self.inter) for t in y]

    def run(self, Qout=None, Kout=None, QKV=None, pages=True):
        self.N.ntp_qk_norm_append_shard(self.shape, self.norm, self.pages if pages else None, self.QKV if QKV is None else QKV, self.dev[0], self.dev[1] if pages else None, self.dev[2],
                                        Qout, Kout)


CASES = [
    # M, q, kv, d, rotary, interleaved, page, pad, far, gammas
    (1, 3, 1, 128, 128, False, 16, 0, 2 ** 31 - 1, "qk"),
    (64, 3, 1, 128, 128, False, 16, 8, 131072, "qk"),
    (257, 14, 14, 128, 128, False, 64, 0, 8192, "qk"),
    (509, 11, 4, 64, 32, True, 32, 40, 1 << 20, "qk"),
    (33, 7, 2, 64, 64, False, 256, 0, 1000, "k"),
    (130, 16, 1, 128, 64, True, 16, 8, 65536, "q"),
    (19, 5, 2, 128, 16, False, 128, 0, 100, ""),
    (40, 4, 3, 64, 0, False, 16, 0, 100, "qk"),
    (4100, 2, 1, 64, 64, True, 64, 0, 5000, "qk"),
    (7, 0, 3, 128, 128, False, 16, 0, 50, "qk"),
    (9, 40, 1, 128, 128, False, 16, 0, 50, "qk"),
]


@pytest.mark.parametrize("fmt", [8, 16])
@pytest.mark.parametrize("M,q,kv,d,rd,inter,page,pad,far,gammas", CASES)
def test_append(M, q, kv, d, rd, inter, page, pad, far, gammas, fmt):
    import torch
    _say(f"qk norm and append, {M} tokens, {q} + {kv} heads of {d}, {rd} rotated, pages of {page}, {fmt} bits")
    c = Case(M, q, kv, d, rd, inter, page, pad, far, gammas, fmt)
    Qout, Kout = _rand(torch, c.g, M, q * d, pad), _rand(torch, c.g, M, kv * d, pad)
    c.run(Qout, Kout)
    torch.cuda.synchronize()
    wQ, wK, wV = c.exact()
    sq, sk = c.sizes()
    for got, want, size in ((Qout, wQ, sq), (Kout, wK, sk)):
        assert (np.abs(f64(got).reshape(want.shape) - want) <= BF * np.abs(want) + 24 * U * size).all()
    there = np.nonzero((c.slots >= 0) & (c.slots < c.n_pages * page))[0]
    at, inside = c.slots[there] // page, c.slots[there] % page
    rest = np.ones((c.n_pages, kv, page), dtype=bool)
    rest[at, :, inside] = False
    if fmt == 16:  # exactly Kout's rows and the values
        K, V = f64(c.both[:, 0]), f64(c.both[:, 1])
        assert np.array_equal(K[at, :, inside], f64(Kout).reshape(M, kv, d)[there]) and np.array_equal(V[at, :, inside], wV[there])
        assert (K[rest] == 9).all() and (V[rest] == 9).all()
    else:
        raw, exps = c.both.cpu().numpy(), c.exps.cpu().numpy().astype(np.int64)
        num = f64(c.both.view(torch.float8_e4m3fn))
        assert (raw[:, 0][rest] == 0x33).all() and (raw[:, 1][rest] == 0x33).all() and (exps[:, 0][rest] == 99).all() and (exps[:, 1][rest] == 99).all()
        # values: bit for bit
        v, code = B.heads_to_8_bits(wV[there])
        assert np.array_equal(exps[:, 1][at, :, inside], code) and np.array_equal(num[:, 1][at, :, inside], v)
        # keys: the power of two of the largest, which may be off by one where that lies next to a border; the numbers next to the keys
        k, size, got = wK[there], sk[there], exps[:, 0][at, :, inside]
        top, slack = np.abs(k).max(-1), 24 * U * size.max(-1)
        assert ((got >= B.e4m3_code(np.maximum(top - slack, 0))) & (got <= B.e4m3_code(top + slack))).all()
        p = np.ldexp(1.0, (got - 127).astype(int))[..., None]
        assert (np.abs(num[:, 0][at, :, inside] * p - k) <= 2.0 ** -4 * np.abs(k) + 2.0 ** -10 * p + 24 * U * size).all()
    if pad:
        assert all(bool(t.as_strided((M, pad), (t.stride(0), 1), t.storage_offset() + t.shape[1]).isnan().all()) for t in (Qout, Kout) if t.shape[1])
    # in place, the queries alone, the pages alone: the same bits
    first, fe = c.both.clone(), None if c.exps is None else c.exps.clone()
    P = c.QKV.clone()
    c.run(P[:, :q * d], P[:, q * d:(q + kv) * d], P)
    assert torch.equal(P[:, :q * d], Qout) and torch.equal(P[:, q * d:(q + kv) * d], Kout) and torch.equal(P[:, (q + kv) * d:], c.QKV[:, (q + kv) * d:])
    Q2 = _rand(torch, c.g, M, q * d)
    c.run(Q2, None, pages=False)
    assert torch.equal(Q2, Qout)
    c.fresh()
    c.run()
    assert torch.equal(c.both, first) and (fe is None or torch.equal(c.exps, fe))


def test_without_norms_it_is_the_append():
    import torch
    import paper_2504_06095_amd as N
    c = Case(200, 5, 3, 128, 64, False, 32, 8, 9999, "", 16)
    Q1, K1, Q2, K2 = (_rand(torch, c.g, 200, n * 128) for n in (5, 3, 5, 3))
    c.run(Q1, K1)
    one = c.both.clone()
    c.fresh()
    N.ntp_kv_append_shard(c.shape, N.kv_cache(c.both[:, 0], c.both[:, 1]), c.QKV, *c.dev, Q2, K2)
    assert torch.equal(Q1, Q2) and torch.equal(K1, K2) and torch.equal(one, c.both)


def test_what_is_not_finite_becomes_nan_alone():
    import torch
    import paper_2504_06095_amd as N
    d, M = 64, 6
    c = Case(M, 1, 2, d, 0, False, 16, 0, 1, "", 8)
    x = c.QKV.view(M, 5, d)
    x[0, 3, 7], x[0, 3, 8], x[1, 4, 0], x[3, 1, 63] = float("inf"), float("nan"), -float("inf"), float("inf")
    x[5, 2] = 3e38
    x[5, 2, 1:] = 1e-37
    c.slots[:] = np.arange(M)
    c.dev = (c.dev[0], torch.arange(M, device="cuda"), None)
    c.run()
    torch.cuda.synchronize()
    num, exps = f64(c.both.view(torch.float8_e4m3fn))[0], c.exps.cpu().numpy()[0]
    t = f64(c.QKV).reshape(M, 5, d)
    for which, first in ((0, 1), (1, 3)):
        want, code = B.heads_to_8_bits(t[:, first:first + 2])
        assert np.array_equal(num[which].transpose(1, 0, 2)[:M], want, equal_nan=True) and np.array_equal(exps[which].T[:M], code)


BWD = [
    # M, q, kv, d, rotary, interleaved, pad, gammas
    (1, 3, 1, 128, 128, False, 0, "qk"),
    (2, 1, 0, 64, 64, False, 0, "qk"),
    (64, 3, 1, 128, 128, False, 8, "qk"),
    (2048, 14, 14, 128, 128, False, 0, "qk"),
    (509, 11, 4, 64, 32, True, 40, "qk"),
    (33, 7, 2, 64, 64, False, 0, "k"),
    (130, 16, 1, 128, 64, True, 8, "q"),
    (19, 5, 2, 128, 16, False, 0, ""),
    (40, 4, 3, 64, 0, False, 0, "qk"),
    (8191, 2, 1, 128, 128, True, 0, "qk"),
    (5, 0, 2, 128, 128, False, 0, "qk"),
]


@pytest.mark.parametrize("workspace", [False, True], ids=["alone", "workspace"])
@pytest.mark.parametrize("M,q,kv,d,rd,inter,pad,gammas", BWD)
def test_gradient(M, q, kv, d, rd, inter, pad, gammas, workspace):
    import torch
    import paper_2504_06095_amd as N
    _say(f"qk norm gradient, {M} tokens, {q} + {kv} heads of {d}, {rd} rotated, {gammas}")
    c = Case(M, q, kv, d, rd, inter, 16, pad, 100000, gammas, 16, seed=1)
    h = N.ntp_create()
    need = N.ntp_workspace_bytes(N.binding.NTP_CALL_QK_NORM, c.shape, handle=h)
    if workspace:
        N.ntp_set_workspace(torch.full((max(need, 256) // 4,), float("nan"), device="cuda"), handle=h)
    dQ, dK = _rand(torch, c.g, M, q * d, pad), _rand(torch, c.g, M, kv * d, pad)
    dQKV = _rand(torch, c.g, M, (q + 2 * kv) * d, pad)
    before = dQKV.clone()
    want, wa, wb = B.qk_norm_bwd(f64(c.QKV), q, kv, d, None if c.gq is None else f64(c.gq), None if c.gk is None else f64(c.gk), EPS, c.pos, c.f, inter, f64(dQ), f64(dK))
    da, db = (torch.full((d,), float("nan"), device="cuda") if t is not None else None for t in (c.gq, c.gk))
    args = (c.shape, c.norm, c.QKV, dQ, dK, c.dev[0], c.dev[2])
    N.ntp_qk_norm_shard_bwd(*args, dQKV, da, db, handle=h)
    torch.cuda.synchronize()
    w = (q + kv) * d
    # sizes of what is added, head by head
    x = f64(c.QKV).reshape(M, -1, d)[:, :q + kv]
    up = np.concatenate([f64(dQ).reshape(M, q, d), f64(dK).reshape(M, kv, d)], 1)
    size = _pairs(np.abs(up), rd, inter)
    tol, sums = np.zeros_like(x), []
    for lo, n, gamma in ((0, q, c.gq), (q, kv, c.gk)):
        sl = slice(lo, lo + n)
        if gamma is None:
            tol[:, sl] = 8 * U * size[:, sl]
            sums.append(None)
            continue
        rstd = 1 / np.sqrt((x[:, sl] ** 2).mean(-1, keepdims=True) + EPS)
        hat, ws = np.abs(x[:, sl]) * rstd, size[:, sl] * np.abs(f64(gamma))
        tol[:, sl] = 64 * U * rstd * (ws + hat * (ws * hat).sum(-1, keepdims=True) / d)
        sums.append((size[:, sl] * hat).sum((0, 1)))
    err = np.abs(f64(dQKV[:, :w]) - want)
    assert (err <= BF * np.abs(want) + tol.reshape(M, -1)).all()
    assert torch.equal(dQKV[:, w:], before[:, w:])
    for got, ref, s in ((da, wa, sums[0]), (db, wb, sums[1])):
        if got is not None:
            assert (np.abs(f64(got) - ref) <= 1e-5 * s).all()
    # the same bits again; added into; in place; without the gammas' gradients
    da2, db2 = (None if t is None else t.clone() for t in (da, db))
    N.ntp_qk_norm_shard_bwd(*args, dQKV, da2, db2, accumulate=True, handle=h)
    for one, two in ((da, da2), (db, db2)):
        assert one is None or torch.equal(one + one, two)
    P = torch.cat([dQ, dK, before[:, w:]], 1)
    da3, db3 = (None if t is None else torch.empty_like(t) for t in (da, db))
    N.ntp_qk_norm_shard_bwd(*args[:3], P[:, :q * d], P[:, q * d:w], *args[5:], P, da3, db3, handle=h)
    assert torch.equal(P, dQKV) and all(a is None or torch.equal(a, b) for a, b in ((da, da3), (db, db3)))
    E = before.clone()
    N.ntp_qk_norm_shard_bwd(*args, E, handle=h)
    assert torch.equal(E, dQKV)
    N.ntp_destroy(h)


def test_no_tokens():
    import torch
    import paper_2504_06095_amd as N
    d = 64
    e = lambda n: torch.empty(0, n * d, dtype=torch.bfloat16, device="cuda")  # noqa: E731
    g = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    shape, norm = N.kv_append_shape(0, dict(q_cnt=2, kv_cnt=1, head_dim=d), 0), N.qk_norm(g, g)
    N.ntp_qk_norm_append_shard(shape, norm, None, e(4), None, None, None, e(2), e(1))
    da, db = torch.full((d,), 5.0, device="cuda"), torch.full((d,), 5.0, device="cuda")
    N.ntp_qk_norm_shard_bwd(shape, norm, e(4), e(2), e(1), None, None, e(4), da, db, accumulate=True)
    assert bool((da == 5).all()) and bool((db == 5).all())
    N.ntp_qk_norm_shard_bwd(shape, norm, e(4), e(2), e(1), None, None, e(4), da, db)
    assert not bool(da.any()) and not bool(db.any())


def test_gradient_against_differences():
    """The gradient that the call gives, along random directions, against differences of the forward call's values in 64 bits on the oracle's side, and its own
    forward call."""
    import torch
    import paper_2504_06095_amd as N
    M, q, kv, d, rd = 5, 3, 2, 64, 32
    c = Case(M, q, kv, d, rd, True, 16, 0, 77, "qk", 16, seed=3)
    c.QKV.copy_(_rand(torch, c.g, M, (q + 2 * kv) * d))
    dQ, dK = _rand(torch, c.g, M, q * d), _rand(torch, c.g, M, kv * d)
    dQKV = torch.zeros(M, (q + 2 * kv) * d, dtype=torch.bfloat16, device="cuda")
    da, db = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    N.ntp_qk_norm_shard_bwd(c.shape, c.norm, c.QKV, dQ, dK, c.dev[0], c.dev[2], dQKV, da, db)
    x, gq, gk, rng = f64(c.QKV), f64(c.gq), f64(c.gk), np.random.default_rng(0)

    def loss(t, a, b):
        Q, K, _ = B.qk_norm(t, q, kv, d, a, b, EPS, c.pos, c.f, True)
        return (Q.reshape(M, -1) * f64(dQ)).sum() + (K.reshape(M, -1) * f64(dK)).sum()

    for _ in range(5):
        t, ta, tb, e = rng.standard_normal(x.shape), rng.standard_normal(d), rng.standard_normal(d), 1e-6
        want = (loss(x + e * t, gq + e * ta, gk + e * tb) - loss(x - e * t, gq - e * ta, gk - e * tb)) / (2 * e)
        got = f64(dQKV)
        parts = [got * t, f64(da) * ta, f64(db) * tb]
        # bf16 steps of the gradient, and 1e-6 of everything for the differences
        assert abs(sum(p.sum() for p in parts) - want) <= BF * np.abs(parts[0]).sum() + 1e-5 * sum(np.abs(p).sum() for p in parts)
