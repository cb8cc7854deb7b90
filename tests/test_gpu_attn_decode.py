"""ntp_attn_decode_shard against the float64 oracle, on a real MI355X.

Tolerance of an output: half a step of bf16 for the result, 2^-8 |C|.  Weights go into the product with the values as bf16 and a bf16 rest (together within
2^-16 of the weight).  fp32: a score is a sum of d products with an error of at most (d + 8) 2^-24 sum |q k| / sqrt(d) (below 2e-4 for the inputs here,
|score| <= 30), which is the relative error of a weight and, with the additions' 2^-24 each, that of the sum: 4e-4 of sum p |V| / sum p, and 4e-4 for LSE."""
import sys

import numpy as np
import pytest

from oracle import block_oracle as B

pytestmark = pytest.mark.gpu
BF, F32 = 2.0 ** -8, 4e-4


def _say(msg):
    print(f"[gpu-case] {msg}", file=sys.stderr, flush=True)


def f64(t):
    return t.double().cpu().numpy()


class Case:
    def __init__(self, lengths, q, kv, d, page, q_off=0, kv_off=0, group=1, max_len=None, seed=0, spare=2, pad=0, q_std=1.5):
        import torch
        import paper_2504_06095_amd as N
        self.torch, self.N, self.lengths, self.q, self.kv, self.d, self.page, self.group = torch, N, list(lengths), q, kv, d, page, group
        g = torch.Generator(device="cuda").manual_seed(seed)
        rng = np.random.default_rng(seed)
        n = len(self.lengths)
        self.max_len = max([0, *self.lengths]) if max_len is None else max_len
        need = [(min(max(x, 0), self.max_len) + page - 1) // page for x in self.lengths]
        cols = (self.max_len + page - 1) // page
        n_pages = sum(need) + spare
        order = rng.permutation(n_pages)
        # what no sequence uses is poisoned: entries behind a sequence's end, pages that nothing names, slots behind the last token
        table = np.full((n, cols + 1), 0x7f000000, dtype=np.int64)
        K, V = (torch.full((n_pages, kv, page, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        at = 0
        for s, k in enumerate(need):
            table[s, :k] = order[at:at + k]
            L = min(max(self.lengths[s], 0), self.max_len)
            for t in (K, V):
                rows = torch.full((k * page, kv, d), float("nan"), device="cuda")
                rows[:L] = torch.randn(L, kv, d, device="cuda", generator=g)
                if k:
                    t[torch.from_numpy(order[at:at + k].copy()).cuda()] = rows.view(k, page, kv, d).transpose(1, 2).to(torch.bfloat16)
            at += k
        self.K, self.V, self.table = K, V, torch.from_numpy(table.astype(np.int32)).cuda()
        self.len_dev = torch.tensor(self.lengths, dtype=torch.int32, device="cuda")
        full = torch.randn(n, q * d + pad, device="cuda", generator=g) * q_std
        self.Q = full.to(torch.bfloat16)[:, :q * d]
        self.plan = dict(q_cnt=q, kv_cnt=kv, q_off=q_off, kv_off=kv_off, head_dim=d)
        self.shape = N.attn_decode_shape(n, self.max_len, self.plan, group)

    def run(self, workspace=False, lse=True):
        torch, N, n = self.torch, self.N, len(self.lengths)
        C = torch.full((n, self.q * self.d + 8), float("nan"), dtype=torch.bfloat16, device="cuda")[:, :self.q * self.d]
        LSE = torch.full((self.q, n), float("nan"), device="cuda") if lse else None
        h = N.ntp_create()
        need = N.ntp_workspace_bytes(N.binding.NTP_CALL_ATTN_DECODE_SHARD, self.shape, handle=h)
        if workspace and need:
            N.ntp_set_workspace(torch.full((need // 4,), float("nan"), device="cuda"), handle=h)
        N.ntp_attn_decode_shard(self.shape, N.kv_cache(self.K, self.V), self.Q, self.table, self.len_dev, C, LSE, handle=h)
        torch.cuda.synchronize()
        N.ntp_destroy(h)
        return C, LSE

    def check(self, C, LSE):
        want, lse, size = B.attn_decode(f64(self.Q), f64(self.K), f64(self.V), self.table.cpu().numpy(), self.lengths, self.max_len, self.plan["q_off"],
                                        self.plan["kv_off"], self.group)
        err = np.abs(f64(C) - want)
        tol = BF * np.abs(want) + F32 * size
        assert (err <= tol).all(), f"C: {np.nanmax(err - tol)} over, {np.isnan(err).sum()} NaN, worst sequence {np.unravel_index((err - tol).argmax(), err.shape)[0]}"
        if LSE is not None:
            e = np.where(np.isneginf(lse) & np.isneginf(f64(LSE)), 0.0, np.abs(f64(LSE) - lse))
            assert (e <= F32).all(), f"LSE: {e.max()}"


CASES = [
    # lengths, q, kv, d, page, q_off, kv_off, group
    ([1], 1, 1, 128, 16, 0, 0, 1),
    ([0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65], 3, 1, 128, 16, 0, 0, 8),
    ([0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129], 11, 4, 64, 32, 11, 2, 4),
    ([-3, 1000, 0, 517], 14, 14, 128, 64, 0, 0, 1),
    ([255, 256, 257, 511, 1025], 32, 2, 128, 256, 0, 0, 16),
    ([700, 3, 299], 5, 2, 64, 16, 3, 0, 6),
    ([2049, 100], 40, 2, 128, 128, 0, 0, 20),
    ([333, 4097], 71, 1, 64, 64, 0, 0, 71),
    ([5000], 8, 8, 128, 1024, 8, 8, 1),
    ([17000], 16, 1, 128, 16, 0, 0, 16),
    ([9001, 1], 3, 2, 64, 16, 7, 1, 4),
]


@pytest.mark.parametrize("workspace", [False, True], ids=["whole", "cut"])
@pytest.mark.parametrize("lengths,q,kv,d,page,q_off,kv_off,group", CASES)
def test_decode(lengths, q, kv, d, page, q_off, kv_off, group, workspace):
    _say(f"decode {lengths}, {q} query heads from {q_off}, {kv} KV heads of {d}, pages of {page}, workspace {workspace}")
    c = Case(lengths, q, kv, d, page, q_off, kv_off, group, seed=len(lengths) + d, pad=8 * (q % 2))
    C, LSE = c.run(workspace)
    c.check(C, LSE)
    again, LSE2 = c.run(workspace)
    assert c.torch.equal(C, again) and c.torch.equal(LSE, LSE2)  # the same bits
    third, _ = c.run(workspace, lse=False)
    assert c.torch.equal(C, third)


@pytest.mark.parametrize("workspace", [False, True], ids=["whole", "cut"])
@pytest.mark.parametrize("d", [64, 128])
def test_lengths_behind_max_len_are_cut(d, workspace):
    c = Case([900, 5000, 64], 4, 2, d, 32, 0, 0, 2, max_len=610)
    c.check(*c.run(workspace))


@pytest.mark.parametrize("lengths", [[5, 0, 300, 1000], [129], [0], [40000, 1, 128, 256, 257] + [7] * 300])
@pytest.mark.parametrize("d", [64, 128])
def test_lengths_far_below_max_len(d, lengths):
    """As in a captured graph: the launch is sized for max_len, and gives what it gives for any other max_len that does not cut them."""
    c = Case(lengths, 5, 2, d, 64, 1, 0, 4, max_len=60000)
    C, LSE = c.run(True)
    c.check(C, LSE)
    c.shape.max_len = max(1, *lengths)
    C1, LSE1 = c.run(False)
    c.check(C1, LSE1)


@pytest.mark.parametrize("q,kv,d,q_off,group", [(5, 2, 128, 1, 4), (5, 2, 64, 1, 4), (40, 2, 64, 0, 20), (1, 1, 128, 3, 16)])
@pytest.mark.parametrize("n", [65, 513, 1300])
def test_many_sequences(n, q, kv, d, q_off, group):
    """More than the 64 and the 512 whose lengths are taken at once, some of them cut by several shares, most of them by none."""
    rng = np.random.default_rng(n + q)
    lengths = rng.integers(0, 150, n)
    for at, length in ((0, 3000), (63, 700), (64, 2100), (n // 2, 5000), (n - 2, 1030), (n - 1, 2500)):
        lengths[at] = length
    c = Case(lengths.tolist(), q, kv, d, 64, q_off, 0, group, max_len=20000, seed=n)
    C, LSE = c.run(True)
    c.check(C, LSE)
    again, LSE2 = c.run(True)
    assert c.torch.equal(C, again) and c.torch.equal(LSE, LSE2)


@pytest.mark.parametrize("workspace", [False, True], ids=["whole", "cut"])
def test_entries_that_name_no_page_are_left_out(workspace):
    c = Case([500, 40, 33, 2000], 6, 3, 128, 16, 0, 0, 2, seed=3)
    c.table[0, 0], c.table[0, 7], c.table[0, 31] = -1, c.K.shape[0], -2 ** 31
    c.table[1, :3] = 2 ** 31 - 1  # a sequence that keeps nothing
    c.table[2, 2] = -5
    c.table[3, 1:] = -1
    c.check(*c.run(workspace))


@pytest.mark.parametrize("workspace", [False, True], ids=["whole", "cut"])
def test_scores_far_apart(workspace):
    """Weights from 1 down to nothing, the largest first, last and in the middle; rows whose scores are all alike; keys whose score is -inf."""
    c = Case([900, 900, 900, 300, 400], 2, 1, 128, 32, 0, 0, 2, q_std=0.0)
    torch = c.torch
    c.Q[:] = 0
    c.Q[:, 0] = 2.0
    c.Q[:, 128] = -2.0
    flat = lambda s, t: (int(c.table[s, t // 32]), 0, t % 32, 0)
    for s, at in ((0, 0), (1, 899), (2, 450)):
        for t in range(900):
            c.K[flat(s, t)] = 80.0 if t == at else -60.0 + (t % 7)
    for t in range(300):
        c.K[flat(3, t)] = 0.0
    for t in range(0, 400, 3):  # head 0: score -inf, head 1: +inf is not asked for
        c.K[flat(4, t)] = float("-inf")
    c.Q[4, 128:] = 0
    c.Q[4, 0] = 1.0
    c.Q[4, 1:128] = 0.5
    C, LSE = c.run(workspace)
    # head 1 of sequence 4 multiplies -inf by 0: NaN by the definition
    assert bool(C[4, 128:].isnan().all()) and bool(LSE[1, 4].isnan())
    c.Q[4, 128:] = c.Q[4, :128]
    C, LSE = c.run(workspace)
    with np.errstate(invalid="ignore"):
        want, lse, size = B.attn_decode(f64(c.Q), f64(c.K), f64(c.V), c.table.cpu().numpy(), c.lengths, c.max_len, 0, 0, 2)
    # the weights of far scores: an fp32 score of size 160 / sqrt(128) * 1.44 = 20 is off by 2^-19, far below F32
    assert (np.abs(f64(C) - want) <= BF * np.abs(want) + F32 * size).all() and (np.abs(f64(LSE) - lse) <= F32).all()


def test_two_handles_on_two_streams():
    """Two batches at once, cut, each on a stream with a handle and a workspace of its own."""
    import torch
    cases = [Case([3000, 17, 900], 8, 2, 128, 16, group=4, seed=1), Case([40, 5000], 6, 3, 64, 32, group=2, seed=2)]
    N = cases[0].N
    torch.cuda.synchronize()
    outs = []
    for c in cases:
        h, st = N.ntp_create(), torch.cuda.Stream()
        with torch.cuda.stream(st):
            need = N.ntp_workspace_bytes(N.binding.NTP_CALL_ATTN_DECODE_SHARD, c.shape, handle=h)
            N.ntp_set_workspace(torch.empty(need, dtype=torch.uint8, device="cuda"), handle=h)
            runs = []
            for _ in range(5):
                C, LSE = torch.empty(len(c.lengths), c.q * c.d, dtype=torch.bfloat16, device="cuda"), torch.empty(c.q, len(c.lengths), device="cuda")
                N.ntp_attn_decode_shard(c.shape, N.kv_cache(c.K, c.V), c.Q, c.table, c.len_dev, C, LSE, handle=h)
                runs.append((C, LSE))
            outs.append((h, runs))
    torch.cuda.synchronize()
    for c, (h, runs) in zip(cases, outs):
        c.check(*runs[0])
        assert all(torch.equal(C, runs[0][0]) and torch.equal(LSE, runs[0][1]) for C, LSE in runs)
        N.ntp_destroy(h)


def test_the_cache_reaches_behind_four_gigabytes():
    import torch
    import paper_2504_06095_amd as N
    d, page, kv, q = 128, 16, 1, 4
    n_pages, stride = 6, 500_000_000  # elements between pages: the last page starts 5 GB into the array
    base = [torch.zeros(stride * (n_pages - 1) + kv * page * d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    K, V = (t.as_strided((n_pages, kv, page, d), (stride, page * d, d, 1)) for t in base)
    small = Case([93, 80], q, kv, d, page, group=4, spare=0, seed=8)
    n = 6
    table = torch.tensor([[5, 0, 3, 1, 4, 2], [4, 2, 5, 0, 1, 0]], dtype=torch.int32, device="cuda")
    for t in (K, V):
        t.copy_(torch.randn(n, kv, page, d, device="cuda"))
    C, LSE = torch.empty(2, q * d, dtype=torch.bfloat16, device="cuda"), torch.empty(q, 2, device="cuda")
    N.ntp_attn_decode_shard(small.shape, N.kv_cache(K, V), small.Q, table, small.len_dev, C, LSE)
    torch.cuda.synchronize()
    small.K, small.V, small.table = K.contiguous(), V.contiguous(), table
    small.check(C, LSE)


def test_no_sequences_and_no_heads():
    import torch
    import paper_2504_06095_amd as N
    K = torch.zeros(2, 1, 16, 64, dtype=torch.bfloat16, device="cuda")
    for n, q in ((0, 3), (2, 0)):
        C = torch.empty(n, q * 64, dtype=torch.bfloat16, device="cuda")
        N.ntp_attn_decode_shard(N.attn_decode_shape(n, 16, dict(q_cnt=q, kv_cnt=1, q_off=0, kv_off=0, head_dim=64), 4), N.kv_cache(K, K), C,
                                torch.zeros(n, 1, dtype=torch.int32, device="cuda"), torch.ones(n, dtype=torch.int32, device="cuda"), C)
    c = Case([0, 0], 3, 1, 128, 16, group=4)
    C, LSE = c.run()
    assert bool((C == 0).all()) and bool((LSE == float("-inf")).all())


def _cut(c, h):
    """A workspace for the call, which the call cuts its work with."""
    need = c.N.ntp_workspace_bytes(c.N.binding.NTP_CALL_ATTN_DECODE_SHARD, c.shape, handle=h)
    assert need > 0
    c.N.ntp_set_workspace(c.torch.full((need // 4,), float("nan"), device="cuda"), handle=h)


@pytest.mark.parametrize("q,kv,d,q_off,group", [(5, 2, 128, 1, 4), (40, 2, 64, 0, 20)])
def test_a_captured_cut_call_serves_every_length(q, kv, d, q_off, group):
    """One capture at a max_len of many steps, replayed with lengths that cut the work differently; eager calls of other lengths and synchronizations between.
    Every replay against the oracle and the eager bits."""
    import torch
    n, top = 70, 20000
    lengths = [top] + [600] * (n - 1)
    c = Case(lengths, q, kv, d, 64, q_off, 0, group, max_len=top, seed=q)
    N = c.N
    # every sequence may reach max_len: those behind the first share its pages
    c.table[1:] = c.table[0]
    h = N.ntp_create()
    _cut(c, h)
    cache = N.kv_cache(c.K, c.V)
    C, LSE = torch.empty(n, q * d, dtype=torch.bfloat16, device="cuda"), torch.empty(q, n, device="cuda")
    run = lambda: N.ntp_attn_decode_shard(c.shape, cache, c.Q, c.table, c.len_dev, C, LSE, handle=h)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            run()
    torch.cuda.synchronize()
    rng = np.random.default_rng(3)
    mixed = rng.integers(0, 3000, n)
    mixed[[7, 64, 69]] = 9000, 0, 19999
    one = np.zeros(n, dtype=np.int64)
    one[65] = top
    for what in (np.full(n, 1), mixed, one, np.full(n, 130), np.zeros(n, dtype=np.int64), mixed[::-1].copy()):
        c.lengths = [int(x) for x in what]
        c.len_dev.copy_(torch.from_numpy(what.astype(np.int32)))
        run()
        torch.cuda.synchronize()
        eager, eager_lse = C.clone(), LSE.clone()
        C.fill_(float("nan"))
        LSE.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(C, eager) and torch.equal(LSE, eager_lse)
        c.check(C, LSE)
    N.ntp_destroy(h)


def test_two_captured_calls_share_a_workspace():
    """Two graphs whose calls use one handle's workspace, replayed in turn on one stream."""
    import torch
    cases = [Case([3000, 17, 900], 8, 2, 128, 16, group=4, seed=1), Case([40, 5000, 2222], 6, 3, 64, 32, group=2, seed=2)]
    N = cases[0].N
    h, st = N.ntp_create(), torch.cuda.Stream()
    need = max(N.ntp_workspace_bytes(N.binding.NTP_CALL_ATTN_DECODE_SHARD, c.shape, handle=h) for c in cases)
    assert need > 0
    N.ntp_set_workspace(torch.full((need // 4,), float("nan"), device="cuda"), handle=h)
    st.wait_stream(torch.cuda.current_stream())
    runs = []
    for c in cases:
        C, LSE = torch.empty(len(c.lengths), c.q * c.d, dtype=torch.bfloat16, device="cuda"), torch.empty(c.q, len(c.lengths), device="cuda")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(st):
            with torch.cuda.graph(graph, stream=st):
                N.ntp_attn_decode_shard(c.shape, N.kv_cache(c.K, c.V), c.Q, c.table, c.len_dev, C, LSE, handle=h)
        runs.append((graph, C, LSE))
    torch.cuda.synchronize()
    with torch.cuda.stream(st):
        for turn in range(3):
            for graph, C, LSE in runs:
                C.fill_(float("nan"))
                LSE.fill_(float("nan"))
            for graph, _, _ in (runs, runs[::-1], runs)[turn]:
                graph.replay()
            torch.cuda.synchronize()
            for c, (_, C, LSE) in zip(cases, runs):
                c.check(C, LSE)
    N.ntp_destroy(h)


@pytest.mark.parametrize("workspace", [False, True], ids=["whole", "cut"])
@pytest.mark.parametrize("d", [64, 128])
def test_lengths_behind_a_max_len_of_many_steps_are_cut(d, workspace):
    c = Case([2900, 5000, 64, 2610], 4, 2, d, 32, 0, 0, 2, max_len=2610)
    h = c.N.ntp_create()
    assert c.N.ntp_workspace_bytes(c.N.binding.NTP_CALL_ATTN_DECODE_SHARD, c.shape, handle=h) > 0
    c.N.ntp_destroy(h)
    c.check(*c.run(workspace))


@pytest.mark.parametrize("workspace", [False, True], ids=["whole", "cut"])
@pytest.mark.parametrize("d", [64, 128])
def test_scores_that_are_all_minus_infinity(d, workspace):
    """A query head that no token counts for gives what a sequence without tokens gives; the heads and sequences beside it are not touched by it."""
    c = Case([1700, 1700, 40], 4, 2, d, 32, 0, 0, 2, max_len=4000)
    C0, LSE0 = c.run(workspace)
    torch = c.torch
    c.Q.view(3, 4, d)[0, :2] = 0.5  # the heads of sequence 0 over KV head 0
    C1, LSE1 = c.run(workspace)
    pages = c.table[0, :(1700 + 31) // 32].long()
    c.K[pages, 0, :, 3] = float("-inf")
    C, LSE = c.run(workspace)
    v, was = C.view(3, 4, d), C1.view(3, 4, d)
    assert bool((v[0, :2] == 0).all()) and bool((LSE[:2, 0] == float("-inf")).all())
    assert torch.equal(v[0, 2:], was[0, 2:]) and torch.equal(v[1:], C0.view(3, 4, d)[1:]) and torch.equal(LSE[:, 1:], LSE0[:, 1:]) and torch.equal(LSE[2:, 0], LSE1[2:, 0])


@pytest.mark.parametrize("workspace", [False, True], ids=["whole", "cut"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [3, 130])
def test_local_kv_heads_that_no_query_head_reads(n, d, workspace):
    """Query heads 12 .. 16 of groups of 4 read global KV heads 3 and 4: the third and fourth of the local ones, which begin at 1."""
    lengths = ([2700, 33, 0, 1500] * n)[:n] if n < 65 else [2700, 33, 0, 1500] + [5, 70] * ((n - 4) // 2)
    c = Case(lengths, 5, 5, d, 32, q_off=12, kv_off=1, group=4, seed=n)
    C, LSE = c.run(workspace)
    c.check(C, LSE)
