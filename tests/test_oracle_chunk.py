"""The oracle of the head norms, the 8-bit cache and the attention of chunks, pinned by closed forms, the e4m3 type of torch, finite differences and the attention of
one new token."""
import numpy as np
import torch

from oracle import block_oracle as B


def test_e4m3_is_torchs_type():
    every = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).float().double().numpy()
    every = every[np.isfinite(every)]
    assert every.max() == 448.0 and np.array_equal(B.to_e4m3(every), every)
    pos = np.sort(every[every >= 0])
    between = np.concatenate([(pos[:-1] + pos[1:]) / 2, pos[:-1] * 0.3 + pos[1:] * 0.7, [1e-9, 447.9, 2.0 ** -10, 3 * 2.0 ** -10]])
    for x in (between, -between):
        assert np.array_equal(B.to_e4m3(x), torch.from_numpy(x).float().to(torch.float8_e4m3fn).float().double().numpy())


def test_power_of_two_of_a_head():
    assert B.e4m3_code([0.0, 448.0, 448.0 * (1 + 1e-12), 1.0, 2.0, 1e-40]).tolist() == [127, 127, 128, 127 - 8, 127 - 7, 16]
    rng = np.random.default_rng(0)
    x = rng.standard_normal((500, 64)) * np.exp(8 * rng.standard_normal((500, 1)))
    q, code = B.heads_to_8_bits(x)
    p = 2.0 ** (code - 127.0)
    assert (np.abs(x).max(1) <= 448 * p).all() and (np.abs(x).max(1) > 224 * p).all()
    assert (np.abs(q * p[:, None] - x) <= 2.0 ** -4 * np.abs(x) + 2.0 ** -10 * p[:, None]).all()
    x[3, 5], x[3, 6] = np.inf, np.nan
    q2, code2 = B.heads_to_8_bits(x)
    assert np.isnan(q2[3, 5:7]).all() and np.isnan(q2).sum() == 2 and np.array_equal(code2[:3], code[:3])


def test_norm_and_its_gradient():
    rng = np.random.default_rng(1)
    M, q, kv, d = 3, 2, 1, 16
    x = rng.standard_normal((M, (q + 2 * kv) * d))
    gq, gk, f, pos, eps = rng.standard_normal(d), rng.standard_normal(d), rng.standard_normal(4), np.array([0, 7, 1000]), 1e-3
    Q, K, V = B.qk_norm(x, q, kv, d, gq, gk, eps, pos, f, False)
    assert np.array_equal(V.reshape(M, -1), x[:, 3 * d:])
    h = x[1, :d]
    assert np.allclose(Q[0, 0], x[0, :d] / np.sqrt((x[0, :d] ** 2).mean() + eps) * gq)  # position 0: not turned
    assert np.isclose((Q[1, 0] ** 2).sum(), ((h * gq) ** 2).sum() / ((h ** 2).mean() + eps))  # lengths are kept
    for gammas in ((gq, gk), (gq, None), (None, None)):
        dQ, dK = rng.standard_normal((M, q * d)), rng.standard_normal((M, kv * d))
        for inter in (False, True):
            def loss(t, a, b):
                Q, K, _ = B.qk_norm(t, q, kv, d, a, b, eps, pos, f, inter)
                return (Q.reshape(M, -1) * dQ).sum() + (K.reshape(M, -1) * dK).sum()
            dx, da, db = B.qk_norm_bwd(x, q, kv, d, *gammas, eps, pos, f, inter, dQ, dK)
            e = 1e-6
            for _ in range(10):
                t = np.zeros_like(x)
                t[:, :3 * d] = rng.standard_normal((M, 3 * d))
                want = (loss(x + e * t, *gammas) - loss(x - e * t, *gammas)) / (2 * e)
                assert abs(want - (dx * t[:, :3 * d]).sum()) < 1e-5
            for i, grad in ((0, da), (1, db)):
                if gammas[i] is None:
                    assert grad is None
                    continue
                t = rng.standard_normal(d)
                moved = [[g if k != i else g + s * e * t for k, g in enumerate(gammas)] for s in (1, -1)]
                assert abs((loss(x, *moved[0]) - loss(x, *moved[1])) / (2 * e) - (grad * t).sum()) < 1e-5


def test_chunks_are_single_tokens_one_after_the_other():
    rng = np.random.default_rng(2)
    pages, kv, page, d, q = 9, 2, 16, 8, 3
    K, V = rng.standard_normal((2, pages, kv, page, d))
    table = np.array([[3, 1, 7], [0, 99, 5], [2, 4, 6]])
    lengths, starts = [41, 37, 3], [0, 5, 5, 10]
    Q = rng.standard_normal((12, q * d))
    C, LSE, A, written = B.attn_chunk(Q, K, V, starts, table, lengths, 100, 48, 1, 0, 2)
    assert written.tolist() == [True] * 10 + [False] * 2
    for s, (lo, hi) in enumerate(zip(starts, starts[1:])):
        for i in range(hi - lo):
            c, l, a = B.attn_decode(Q[lo + i:lo + i + 1], K, V, table[s:s + 1], [lengths[s] - (hi - lo) + i + 1], 48, 1, 0, 2)
            assert np.allclose(C[lo + i], c[0]) and np.allclose(A[lo + i], a[0]) and np.array_equal(np.isneginf(LSE[:, lo + i]), np.isneginf(l[:, 0]))
    assert not C[5:7].any() and np.isneginf(LSE[:, 5:7]).all() and C[7:10].any()  # three tokens under five rows: the first two see none
    one, _, _, _ = B.attn_chunk(Q[:3], K, V, None, table, lengths, 1, 48, 1, 0, 2)
    assert np.allclose(one, B.attn_decode(Q[:3], K, V, table, lengths, 48, 1, 0, 2)[0])
    few, _, _, w = B.attn_chunk(Q, K, V, starts, table, lengths, 2, 48, 1, 0, 2)
    assert w.tolist() == [True] * 2 + [False] * 3 + [True] * 2 + [False] * 5 and np.allclose(few[:2], C[:2]) and not few[2:].any()
