"""ntp_attn_chunk_shard against the float64 oracle, on a real MI355X, over bf16 and 8-bit pages.

Tolerance of an output: half a step of bf16 for the result, 2^-8 |C|.  A weight goes into the product with the values as bf16: half a step, 2^-8 of sum p |V| / sum p at most.
fp32: a score is a sum of d products with an error of at most (d + 8) 2^-24 sum |q k| / sqrt(d) (below 2e-4 for the inputs here, |score| <= 30), which is the
relative error of a weight and, with the additions' 2^-24 each, that of the sum: 4e-4 of sum p |V| / sum p, and 4e-4 for LSE.  8-bit keys and values are exact in bf16."""
import sys

import numpy as np
import pytest

from oracle import block_oracle as B

pytestmark = pytest.mark.gpu
BF, F32 = 2.0 ** -8, 4e-4


def _say(msg):
    print(f"[gpu-case] {msg}", file=sys.stderr, flush=True)


def f64(t):
    return t.float().double().cpu().numpy()


class Case:
    def __init__(self, news, lengths, q, kv, d, page, q_off=0, kv_off=0, group=1, fmt=16, max_len=None, max_new=None, seed=0, spare=2, pad=0, padded=0, single=False, q_std=1.5,
                 lead=0, bad=False):
        import torch
        import paper_2504_06095_amd as N
        self.torch, self.N, self.news, self.lengths, self.q, self.kv, self.d, self.page, self.group, self.fmt = torch, N, list(news), list(lengths), q, kv, d, page, group, fmt
        g = torch.Generator(device="cuda").manual_seed(seed)
        rng = np.random.default_rng(seed)
        n = len(self.lengths)
        self.max_len = max([0, *self.lengths]) if max_len is None else max_len
        self.max_new = max([0, *self.news]) if max_new is None else max_new
        need = [(min(max(x, 0), self.max_len) + page - 1) // page for x in self.lengths]
        cols = (self.max_len + page - 1) // page
        n_pages = sum(need) + spare
        order = rng.permutation(n_pages)
        # what no sequence uses is poisoned: entries behind a sequence's end, pages that nothing names, slots behind the last token
        table = np.full((n, cols + 1), 0x7f000000, dtype=np.int64)
        K, V = (torch.full((n_pages, kv, page, d), float("nan"), device="cuda") for _ in range(2))
        at = 0
        for s, k in enumerate(need):
            table[s, :k] = order[at:at + k]
            if bad and k > 2:  # pages that do not exist
                table[s, 1], table[s, k - 1] = -5, n_pages
            L = min(max(self.lengths[s], 0), self.max_len)
            for t in (K, V):
                rows = torch.full((k * page, kv, d), float("nan"), device="cuda")
                rows[:L] = torch.randn(L, kv, d, device="cuda", generator=g) * torch.exp(0.4 * torch.randn(L, kv, 1, device="cuda", generator=g)).clamp(max=2.0)
                if k:
                    t[torch.from_numpy(order[at:at + k].copy()).cuda()] = rows.view(k, page, kv, d).transpose(1, 2)
            at += k
        if fmt == 16:
            self.K, self.V = K.bfloat16(), V.bfloat16()
            self.pages = N.kv_pages(self.K, self.V)
            self.numbers = f64(self.K), f64(self.V)
        else:
            self.raw, self.numbers = [], []
            for t in (K, V):
                top = t.nan_to_num(0).abs().amax(-1)
                part, e = torch.frexp(top)
                code = torch.where(top == 0, 0xff, (e - 9 + (part > 0.875) + 127))  # (0xff and NaN numbers where nothing is)
                num = torch.ldexp(t, 127 - code[..., None].float()).to(torch.float8_e4m3fn)
                self.raw += [num, code.to(torch.uint8)]
                self.numbers.append(np.ldexp(f64(num), (code.cpu().numpy() - 127)[..., None]))
            self.pages = N.kv_pages(self.raw[0], self.raw[2], self.raw[1], self.raw[3])
        self.table = torch.from_numpy(table.astype(np.int32)).cuda()
        self.len_dev = torch.tensor(self.lengths, dtype=torch.int32, device="cuda")
        self.starts = None if single else [lead + int(x) for x in np.concatenate([[0], np.cumsum(self.news)])]
        self.M = n if single else self.starts[-1] + padded
        self.starts_dev = None if single else torch.tensor(self.starts, dtype=torch.int32, device="cuda")
        full = torch.randn(self.M, q * d + pad, device="cuda", generator=g) * q_std
        self.Q = full.to(torch.bfloat16)[:, :q * d]
        self.plan = dict(q_cnt=q, kv_cnt=kv, q_off=q_off, kv_off=kv_off, head_dim=d)
        self.shape = N.attn_chunk_shape(self.M, n, self.max_new, self.max_len, self.plan, group)

    def run(self, workspace=False, lse=True):
        torch, N = self.torch, self.N
        C = torch.full((self.M, self.q * self.d + 8), 77.0, dtype=torch.bfloat16, device="cuda")[:, :self.q * self.d]
        LSE = torch.full((self.q, self.M), 77.0, device="cuda") if lse else None
        h = N.ntp_create()
        need = N.ntp_workspace_bytes(N.binding.NTP_CALL_ATTN_CHUNK_SHARD, self.shape, handle=h)
        if workspace and need:
            N.ntp_set_workspace(torch.full((need // 4,), float("nan"), device="cuda"), handle=h)
        N.ntp_attn_chunk_shard(self.shape, self.pages, self.Q, self.starts_dev, self.table, self.len_dev, C, LSE, handle=h)
        torch.cuda.synchronize()
        N.ntp_destroy(h)
        return C, LSE

    def check(self, C, LSE):
        want, lse, size, written = B.attn_chunk(f64(self.Q), *self.numbers, self.starts, self.table.cpu().numpy(), self.lengths, self.max_new, self.max_len,
                                                self.plan["q_off"], self.plan["kv_off"], self.group)
        got = f64(C)
        assert (got[~written] == 77).all(), "rows of no sequence have been written"
        err = np.abs(got - want)[written]
        tol = (BF * np.abs(want) + (BF + F32) * size)[written]
        assert (err <= tol).all(), f"C: {np.nanmax(err - tol)} over, {np.isnan(err).sum()} NaN, {(~(err <= tol)).sum()} wrong, first {np.argwhere(~(err <= tol))[0]}"
        if LSE is not None:
            l = f64(LSE)
            assert (l[:, ~written] == 77).all()
            l, lse = l[:, written], lse[:, written]
            e = np.where(np.isneginf(lse) & np.isneginf(l), 0.0, np.abs(l - lse))
            assert (e <= F32).all(), f"LSE: {np.nanmax(e)}"


CASES = [
    # new tokens, lengths, q, kv, d, page, q_off, kv_off, group
    ([1], [1], 1, 1, 128, 16, 0, 0, 1),
    ([2, 3, 1, 0, 5], [2, 30, 17, 64, 5], 3, 1, 128, 16, 0, 0, 8),
    ([4] * 6, [4, 5, 64, 65, 257, 1023], 8, 1, 128, 16, 8, 1, 8),
    ([1, 1, 1, 1], [0, 1, 16, 600], 11, 4, 64, 32, 11, 2, 4),
    ([130, 1, 0, 17], [130, 900, 3, 1000], 14, 14, 128, 64, 0, 0, 1),
    ([64, 63, 65, 128, 127, 129], [64, 63, 65, 128, 127, 129], 2, 2, 64, 16, 0, 0, 1),
    ([5, 40, 7], [3, 20, 0], 4, 2, 128, 16, 0, 0, 2),          # shorter than their rows: the first see nothing
    ([33, 1, 300], [333, 700, 1300], 11, 4, 64, 32, 11, 2, 4),
    ([257], [2049], 32, 2, 128, 256, 0, 0, 16),
    ([3, 20], [700, 299], 5, 2, 64, 16, 3, 0, 6),
    ([9, 1], [333, 4097], 71, 1, 64, 64, 0, 0, 71),
    ([600], [600], 6, 3, 128, 1024, 6, 3, 2),
    ([16, 1, 1], [9001, 1, 5000], 3, 2, 64, 16, 7, 1, 4),
    ([1, 500, 1, 2, 1], [2000, 1500, 30, 3000, 1], 16, 2, 128, 64, 0, 0, 8),
    ([1] * 70 + [40], [7 * i % 300 for i in range(70)] + [100], 4, 1, 64, 16, 0, 0, 4),
]


@pytest.mark.parametrize("fmt", [16, 8])
@pytest.mark.parametrize("workspace", [False, True], ids=["whole", "cut"])
@pytest.mark.parametrize("news,lengths,q,kv,d,page,q_off,kv_off,group", CASES)
def test_chunks(news, lengths, q, kv, d, page, q_off, kv_off, group, workspace, fmt):
    _say(f"chunks {news} of {lengths}, {q} query heads from {q_off}, {kv} KV heads of {d}, pages of {page}, {fmt} bits, workspace {workspace}")
    c = Case(news, lengths, q, kv, d, page, q_off, kv_off, group, fmt, seed=len(lengths) + d, pad=8 * (q % 2), padded=3 * (q % 2), lead=2 * (q % 3 == 0))
    C, LSE = c.run(workspace)
    c.check(C, LSE)
    again, LSE2 = c.run(workspace)
    assert c.torch.equal(C, again) and c.torch.equal(LSE, LSE2)  # the same bits
    third, _ = c.run(workspace, lse=False)
    assert c.torch.equal(C, third)


@pytest.mark.parametrize("fmt", [16, 8])
@pytest.mark.parametrize("workspace", [False, True], ids=["whole", "cut"])
@pytest.mark.parametrize("lengths,q,kv,d,page,group", [([0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129], 3, 1, 128, 16, 8), ([17000], 16, 1, 128, 16, 16), ([-3, 1000, 0, 517], 14, 14, 64, 64, 1),
                                                       ([2049, 100], 40, 2, 128, 128, 20), ([255, 256, 257, 511, 1025], 32, 2, 64, 256, 16)])
def test_one_token_of_each_sequence(lengths, q, kv, d, page, group, workspace, fmt):
    c = Case([1] * len(lengths), lengths, q, kv, d, page, 0, 0, group, fmt, seed=d, single=True)
    C, LSE = c.run(workspace)
    c.check(C, LSE)
    c.starts_dev = c.torch.arange(c.M + 1, dtype=c.torch.int32, device="cuda")
    same, _ = c.run(workspace)
    assert c.torch.equal(C, same)


@pytest.mark.parametrize("fmt", [16, 8])
@pytest.mark.parametrize("workspace", [False, True], ids=["whole", "cut"])
@pytest.mark.parametrize("d", [64, 128])
def test_what_passes_the_bounds_is_cut(d, workspace, fmt):
    c = Case([3, 90, 20], [900, 5000, 64], 4, 2, d, 32, 0, 0, 2, fmt, max_len=610, max_new=50)
    c.check(*c.run(workspace))


@pytest.mark.parametrize("fmt", [16, 8])
@pytest.mark.parametrize("workspace", [False, True], ids=["whole", "cut"])
@pytest.mark.parametrize("news,lengths", [([1, 1], [300, 77]), ([40, 200], [3000, 400])])
def test_pages_that_do_not_exist_are_left_out(news, lengths, workspace, fmt):
    c = Case(news, lengths, 4, 2, 128, 16, 0, 0, 2, fmt, bad=True)
    c.check(*c.run(workspace))


@pytest.mark.parametrize("fmt", [16, 8])
@pytest.mark.parametrize("workspace", [False, True], ids=["whole", "cut"])
def test_bounds_far_above_the_batch(workspace, fmt):
    c = Case([1, 70, 0, 300, 9], [5, 100, 300, 1000, 2000], 8, 2, 128, 16, 0, 0, 4, fmt, max_len=200000, max_new=4096, padded=900)
    c.check(*c.run(workspace))


@pytest.mark.parametrize("workspace", [False, True], ids=["whole", "cut"])
@pytest.mark.parametrize("news,lengths", [([1] * 5, [300] * 5), ([100, 3], [800, 300])])
def test_scores_that_are_all_minus_infinity_give_zeros(news, lengths, workspace):
    import torch
    c = Case(news, lengths, 2, 1, 64, 16, 0, 0, 2, 16)
    c.K.copy_(torch.where(c.K.isnan(), c.K, torch.full_like(c.K, -float("inf"))))
    c.Q.copy_(c.Q.abs() + 0.125)
    C, LSE = c.run(workspace)
    assert not bool(C.any()) and bool(torch.isneginf(LSE).all())


def test_starts_outside_the_rows_are_taken_to_the_nearer_end():
    import torch
    c = Case([20, 30], [200, 300], 2, 1, 64, 16, 0, 0, 2, 16)
    c.starts = [-7, 20, 5000]
    c.starts_dev = torch.tensor(c.starts, dtype=torch.int32, device="cuda")
    c.max_new = 50
    c.shape = c.N.attn_chunk_shape(c.M, 2, 50, c.max_len, c.plan, 2)
    c.check(*c.run(True))


def test_nothing_to_do():
    import torch
    import paper_2504_06095_amd as N
    e = torch.empty(0, 1, 16, 64, dtype=torch.bfloat16, device="cuda")
    plan = dict(q_cnt=2, kv_cnt=1, q_off=0, kv_off=0, head_dim=64)
    z = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    for M, n, new in ((0, 0, 4), (3, 0, 4), (3, 1, 0)):
        Q, C = (torch.full((M, 128), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        N.ntp_attn_chunk_shard(N.attn_chunk_shape(M, n, new, 0, plan, 2), N.kv_pages(e, e), Q, z(n + 1), z(n, 0), z(n), C)
        assert bool((C == 5).all())
    Q, C = (torch.full((3, 128), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    N.ntp_attn_chunk_shard(N.attn_chunk_shape(3, 1, 3, 40, plan, 2), N.kv_pages(e, e), Q, torch.tensor([0, 3], dtype=torch.int32, device="cuda"), z(1, 3), z(1) + 40, C)
    assert not bool(C.any())  # a cache without pages: no row sees anything


@pytest.mark.parametrize("fmt", [16, 8])
@pytest.mark.parametrize("length", [448, 449, 503, 511, 512, 513, 961, 1023, 1024, 1025])
def test_whole_walks_around_the_lengths_of_their_levels(length, fmt):
    """Walks are taken longest first by levels of 512 tokens: max_len just below, at and behind a level's border (below it the highest level once had no walks looked for, and row
    tiles came out of the lengths' range)."""
    _say(f"whole walks, 9 sequences of {length}, {fmt} bits")
    c = Case([length - 6] * 9, [length] * 9, 4, 4, 128, 16, 0, 0, 1, fmt)
    c.check(*c.run(False))
    c.check(*c.run(True))


@pytest.mark.parametrize("fmt,d", [(16, 64), (8, 128)])
def test_more_whole_walks_than_places(fmt, d):
    news = [600, 130, 33, 511, 640, 129, 577, 600, 1, 600]
    lengths = [600, 200, 700, 511, 1000, 129, 700, 640, 30, 1100]
    c = Case(news, lengths, 15, 5, d, 64, 1, 0, 4, fmt, padded=3) if d == 64 else Case(news, lengths, 14, 14, d, 64, 0, 0, 1, fmt, padded=3)
    c.check(*c.run(True))


@pytest.mark.parametrize("fmt", [16, 8])
@pytest.mark.parametrize("workspace", [False, True], ids=["whole", "cut"])
@pytest.mark.parametrize("long_ones", [1, 40])
def test_hundreds_of_sequences(long_ones, workspace, fmt):
    rng = np.random.default_rng(7)
    n = 700
    news, lengths = [1] * n, [int(x) for x in rng.integers(0, 90, n)]
    for i in rng.choice(n, long_ones, replace=False):
        news[i] = int(rng.integers(33, 150))
        lengths[i] = news[i] + int(rng.integers(0, 1200 if long_ones > 1 else 5000))
    _say(f"{n} sequences, {long_ones} of them with chunks, {fmt} bits")
    c = Case(news, lengths, 2, 1, 64, 16, 0, 0, 2, fmt)
    c.check(*c.run(workspace))


@pytest.mark.parametrize("parts", [1, 2, 5, 16])
def test_parts_by_option(parts):
    import torch
    c = Case([200, 1, 77], [1500, 300, 2100], 6, 2, 128, 32, 0, 0, 3, 16)
    want, _ = c.run(True)
    N, h = c.N, c.N.ntp_create()
    N.ntp_set_option(N.binding.NTP_OPT_ATTN_PARTS, parts, handle=h)
    N.ntp_set_workspace(torch.empty(N.ntp_workspace_bytes(N.binding.NTP_CALL_ATTN_CHUNK_SHARD, c.shape, handle=h), dtype=torch.uint8, device="cuda"), handle=h)
    C, LSE = torch.full_like(want, 77.0), torch.full((6, c.M), 77.0, device="cuda")
    N.ntp_attn_chunk_shard(c.shape, c.pages, c.Q, c.starts_dev, c.table, c.len_dev, C, LSE, handle=h)
    torch.cuda.synchronize()
    c.check(C, LSE)
    N.ntp_destroy(h)


@pytest.mark.parametrize("fmt", [16, 8])
def test_pages_behind_four_gigabytes(fmt):
    """Keys and values of 5.4 GB (bf16) and 2.7 GB (8 bits, 43 MB of powers of two); the batch's pages are the last ones."""
    import torch
    import paper_2504_06095_amd as N
    d, page, kv, n_pages = 128, 4096, 2, 2570
    K, V = (torch.zeros(n_pages, kv, page, d, dtype=torch.bfloat16 if fmt == 16 else torch.uint8, device="cuda") for _ in range(2))
    E = [torch.full((n_pages, kv, page), 127, dtype=torch.uint8, device="cuda") for _ in range(2)] if fmt == 8 else []
    plan, f8 = dict(q_cnt=6, kv_cnt=kv, q_off=0, kv_off=0, head_dim=d), torch.float8_e4m3fn
    pages = N.kv_pages(K, V) if fmt == 16 else N.kv_pages(K.view(f8), V.view(f8), *E)
    news, lens = [1, 200, 40], [700, 4100, 40]
    table = torch.tensor([[n_pages - 1, 0], [n_pages - 2, n_pages - 4], [n_pages - 3, 0]], dtype=torch.int32, device="cuda")
    tokens = [(s, t) for s, n in enumerate(lens) for t in range(n)]
    slots = torch.tensor([int(table[s, t // page]) * page + t % page for s, t in tokens], device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    QKV = torch.randn(len(tokens), 10 * d, device="cuda", generator=g).bfloat16()
    N.ntp_qk_norm_append_shard(N.kv_append_shape(len(tokens), plan, 0), None, pages, QKV, None, slots, None)
    M = sum(news)
    Q = torch.randn(M, 6 * d, device="cuda", generator=g).bfloat16()
    starts, L = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 1, 201, 241], lens))
    C, h = torch.zeros(M, 6 * d, dtype=torch.bfloat16, device="cuda"), N.ntp_create()
    shape = N.attn_chunk_shape(M, 3, 200, 4100, plan, 3)
    N.ntp_set_workspace(torch.empty(N.ntp_workspace_bytes(N.binding.NTP_CALL_ATTN_CHUNK_SHARD, shape, handle=h), dtype=torch.uint8, device="cuda"), handle=h)
    N.ntp_attn_chunk_shard(shape, pages, Q, starts, table, L, C, handle=h)
    torch.cuda.synchronize()
    assert int((K != 0).any(3).sum()) == kv * len(tokens)
    # the oracle over the few pages in use
    used = torch.tensor([n_pages - 4, n_pages - 3, n_pages - 2, n_pages - 1], device="cuda")
    num = [f64(t[used]) if fmt == 16 else np.ldexp(f64(t[used].view(f8)), (e[used].cpu().numpy().astype(np.int64) - 127)[..., None]) for t, e in zip((K, V), E or (None, None))]
    small = np.array([[3, 0], [2, 0], [1, 0]])
    want, _, size, _ = B.attn_chunk(f64(Q), *num, [0, 1, 201, 241], small, lens, 200, 4100, 0, 0, 3)
    assert (np.abs(f64(C) - want) <= BF * np.abs(want) + (BF + F32) * size).all()
    N.ntp_destroy(h)


@pytest.mark.parametrize("new", [1, 50])
def test_a_batch_without_any_tokens(new):
    import torch
    import paper_2504_06095_amd as N
    e = torch.empty(0, 1, 16, 64, dtype=torch.bfloat16, device="cuda")
    plan = dict(q_cnt=2, kv_cnt=1, q_off=0, kv_off=0, head_dim=64)
    z = lambda *s: torch.zeros(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    M = 2 * new
    C, LSE = torch.full((M, 128), 5.0, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, M, device="cuda")
    N.ntp_attn_chunk_shard(N.attn_chunk_shape(M, 2, new, 0, plan, 2), N.kv_pages(e, e), torch.ones_like(C), torch.tensor([0, new, M], dtype=torch.int32, device="cuda"), z(2, 0), z(2), C, LSE)
    assert not bool(C.any()) and bool(torch.isneginf(LSE).all())


def test_a_call_ends_with_the_rows_that_it_has():
    """Views of wider matrices, with what lies beside the columns left alone."""
    import torch
    c = Case([70, 1, 33], [400, 90, 33], 5, 2, 64, 16, 3, 0, 6, 8, pad=24)
    full = torch.full((c.M + 2, 5 * 64 + 40), 77.0, dtype=torch.bfloat16, device="cuda")
    C = full[1:-1, 16:16 + 5 * 64]
    c.N.ntp_attn_chunk_shard(c.shape, c.pages, c.Q, c.starts_dev, c.table, c.len_dev, C)
    torch.cuda.synchronize()
    c.check(C, None)
    full[1:-1, 16:16 + 5 * 64] = 77.0
    assert bool((full == 77).all())
