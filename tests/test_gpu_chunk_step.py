"""The head norms, the pages of either format and the attention of chunks together, as a user runs them, on a real MI355X: batches whose sequences each bring a chunk of a prompt, a few
proposed tokens, one or none; the same from captured graphs; and the gradient's way through the attention core and the norms.

The attention is compared with the float64 oracle over the queries and the pages that the append wrote (tolerance as tests/test_gpu_attn_chunk.py); what the append wrote with one call
for all tokens, bit for bit."""
import sys

import numpy as np
import pytest

from oracle import block_oracle as B

pytestmark = pytest.mark.gpu
BF, F32, EPS = 2.0 ** -8, 4e-4, 1e-6


def _say(msg):
    print(f"[gpu-case] {msg}", file=sys.stderr, flush=True)


def f64(t):
    return t.float().double().cpu().numpy()


class Server:
    """One rank's attention of a few sequences, from their QKV rows on."""

    def __init__(self, tokens, n_q, n_kv, d, tp, rank, page, fmt, seed=0, handle=None, spare=0):
        import torch
        import paper_2504_06095_amd as N
        self.torch, self.N, self.d, self.page, self.fmt = torch, N, d, page, fmt
        self.plan, self.group = N.ntp_attn_shard_plan(n_q, n_kv, d, tp, rank), n_q // n_kv
        p, g = self.plan, torch.Generator(device="cuda").manual_seed(seed)
        self.q, self.kv = p["q_cnt"], p["kv_cnt"]
        self.QKV = [torch.randn(t, p["w_qkv"], device="cuda", generator=g).bfloat16() for t in tokens]
        self.gq, self.gk = ((1 + 0.2 * torch.randn(d, device="cuda", generator=g)).bfloat16() for _ in range(2))
        self.norm = N.qk_norm(self.gq, self.gk, EPS)
        self.inv_freq = torch.tensor([10000.0 ** (-2 * i / d) for i in range(d // 2)], dtype=torch.float64, device="cuda")
        self.n, self.most = len(tokens), max(tokens)
        per_seq = (self.most + page - 1) // page
        n_pages = self.n * per_seq + 2
        self.table = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed))[:self.n * per_seq].view(self.n, per_seq)
        self.table_d = self.table.to(torch.int32).cuda()
        self.kv_tensors = self.new_pages(n_pages)
        self.pages = N.kv_pages(*self.kv_tensors)
        self.at = [0] * self.n
        self.h = handle or N.ntp_create()

    def new_pages(self, n):
        torch = self.torch
        shape = (n, self.kv, self.page, self.d)
        if self.fmt == 16:
            return [torch.full(shape, float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        return ([torch.full(shape, 0x7f, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2)]
                + [torch.full(shape[:3], 0xff, dtype=torch.uint8, device="cuda") for _ in range(2)])

    def slot(self, s, t):
        return int(self.table[s, t // self.page]) * self.page + t % self.page

    def batch(self, news, rows):
        """Device inputs of a batch of `rows` rows, those behind the sequences' padding."""
        torch = self.torch
        x = torch.full((rows, self.plan["w_qkv"]), 3.0, dtype=torch.bfloat16, device="cuda")
        pos, slots, starts, lengths, at = [0] * rows, [-1] * rows, [0], [], 0
        for s, n in enumerate(news):
            t0 = self.at[s]
            x[at:at + n] = self.QKV[s][t0:t0 + n]
            for i in range(n):
                pos[at + i], slots[at + i] = t0 + i, self.slot(s, t0 + i)
            at += n
            starts.append(at)
            lengths.append(t0 + n)
        dev = lambda v, t: torch.tensor(v, dtype=t, device="cuda")  # noqa: E731
        return dict(x=x, pos=dev(pos, torch.int32), slots=dev(slots, torch.int64), starts=dev(starts, torch.int32), lengths=dev(lengths, torch.int32), host=(starts, lengths))

    def buffers(self, rows):
        e = lambda w: self.torch.full((rows, w), 7.0, dtype=self.torch.bfloat16, device="cuda")  # noqa: E731
        return dict(Q=e(self.q * self.d), C=e(self.q * self.d))

    def shapes(self, rows, max_new):
        N = self.N
        a, c = N.kv_append_shape(rows, self.plan), N.attn_chunk_shape(rows, self.n, max_new, self.most, self.plan, self.group)
        need = N.ntp_workspace_bytes(N.binding.NTP_CALL_ATTN_CHUNK_SHARD, c, handle=self.h)
        return a, c, need

    def run(self, shapes, b, o):
        N = self.N
        N.ntp_qk_norm_append_shard(shapes[0], self.norm, self.pages, b["x"], b["pos"], b["slots"], self.inv_freq, o["Q"], handle=self.h)
        N.ntp_attn_chunk_shard(shapes[1], self.pages, o["Q"], b["starts"], self.table_d, b["lengths"], o["C"], handle=self.h)

    def numbers(self):
        if self.fmt == 16:
            return [f64(t) for t in self.kv_tensors]
        return [np.ldexp(f64(t), (e.cpu().numpy().astype(np.int64) - 127)[..., None]) for t, e in zip(self.kv_tensors[:2], self.kv_tensors[2:])]

    def check(self, b, o, max_new):
        starts, lengths = b["host"]
        want, _, size, written = B.attn_chunk(f64(o["Q"]), *self.numbers(), starts, self.table.numpy(), lengths, max_new, self.most, self.plan["q_off"], self.plan["kv_off"], self.group)
        got = f64(o["C"])
        assert (np.abs(got - want)[written] <= (BF * np.abs(want) + (BF + F32) * size)[written]).all() and (got[~written] == 7).all()


# the new tokens of three sequences, step by step
STEPS = [(40, 0, 129), (1, 64, 3), (1, 1, 1), (200, 4, 0), (0, 33, 2), (7, 1, 300), (1, 150, 1)]


@pytest.mark.parametrize("fmt", [16, 8])
@pytest.mark.parametrize("n_q,n_kv,d,tp,rank,page", [(16, 4, 64, 3, 1, 16), (16, 16, 128, 7, 0, 64), (16, 2, 128, 8, 7, 32)])
def test_batches_of_chunks(n_q, n_kv, d, tp, rank, page, fmt):
    import torch
    _say(f"batches of chunks, heads {n_q} / {n_kv} of {d} at TP {tp} rank {rank}, {fmt} bits")
    tokens = [sum(s[i] for s in STEPS) for i in range(3)]
    S = Server(tokens, n_q, n_kv, d, tp, rank, page, fmt)
    rows, max_new = max(sum(s) for s in STEPS) + 5, 300
    shapes, o = S.shapes(rows, max_new), S.buffers(rows)
    if shapes[2]:
        S.N.ntp_set_workspace(torch.empty(shapes[2], dtype=torch.uint8, device="cuda"), handle=S.h)
    for news in STEPS:
        b = S.batch(news, rows)
        o["C"].fill_(7.0)
        S.run(shapes, b, o)
        torch.cuda.synchronize()
        for s, n in enumerate(news):
            S.at[s] += n
        S.check(b, o, max_new)
    # the pages: as one call for all tokens leaves them
    T = Server(tokens, n_q, n_kv, d, tp, rank, page, fmt)
    b = T.batch(tokens, sum(tokens))
    T.N.ntp_qk_norm_append_shard(T.N.kv_append_shape(sum(tokens), T.plan), T.norm, T.pages, b["x"], b["pos"], b["slots"], T.inv_freq, None)
    torch.cuda.synchronize()
    for x, y in zip(S.kv_tensors, T.kv_tensors):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    # both kinds of call on one cache
    if fmt == 16:
        L = torch.tensor(tokens, dtype=torch.int32, device="cuda")
        one, two = S.buffers(3)["C"], S.buffers(3)["C"]
        Q = torch.randn(3, S.q * d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)).bfloat16()
        S.N.ntp_attn_decode_shard(S.N.attn_decode_shape(3, S.most, S.plan, S.group), S.N.kv_cache(*S.kv_tensors), Q, S.table_d, L, one)
        S.N.ntp_attn_chunk_shard(S.N.attn_chunk_shape(3, 3, 1, S.most, S.plan, S.group), S.pages, Q, None, S.table_d, L, two)
        torch.cuda.synchronize()
        assert (np.abs(f64(one) - f64(two)) <= 4 * BF * np.abs(f64(one)) + 4e-3).all()
    S.N.ntp_destroy(S.h)
    T.N.ntp_destroy(T.h)


@pytest.mark.parametrize("fmt", [16, 8])
def test_two_captured_steps_share_a_workspace(fmt):
    """One graph of batches with chunks, one of single tokens, on one handle and workspace, replayed in turn with other lengths, and eager calls between them."""
    import torch
    import paper_2504_06095_amd as N
    tokens = [700, 300, 450]
    S = Server(tokens, 16, 4, 128, 3, 1, 16, fmt, seed=5)
    rows = 420
    big, small = S.shapes(rows, 300), S.shapes(3, 1)
    ws = torch.full((max(big[2], small[2], 4) // 4,), float("nan"), device="cuda")
    N.ntp_set_workspace(ws, handle=S.h)
    ob, os_ = S.buffers(rows), S.buffers(3)
    ib, is_ = S.batch((200, 1, 30), rows), S.batch((1, 1, 1), 3)
    side = torch.cuda.Stream()
    S.run(big, ib, ob)  # (kernels are loaded before the capture)
    S.run(small, is_, os_)
    torch.cuda.synchronize()
    graphs = []
    for shapes, i, o in ((big, ib, ob), (small, is_, os_)):
        g = torch.cuda.CUDAGraph()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            with torch.cuda.graph(g, stream=side):
                S.run(shapes, i, o)
        torch.cuda.synchronize()
        graphs.append(g)

    def put(into, b):
        for k in ("x", "pos", "slots", "starts", "lengths"):
            into[k].copy_(b[k])

    for news in ((200, 1, 30), (1, 1, 1), (299, 40, 2), (1, 1, 1), (1, 1, 1), (3, 120, 200)):
        single = news == (1, 1, 1)
        shapes, i, o, g, n = (small, is_, os_, graphs[1], 3) if single else (big, ib, ob, graphs[0], rows)
        b = S.batch(news, n)
        put(i, b)
        o["C"].fill_(7.0)
        ws.fill_(float("nan"))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        got = o["C"].clone()
        for s, k in enumerate(news):
            S.at[s] += k
        i["host"] = b["host"]
        S.check(dict(b), dict(Q=o["Q"], C=got), 1 if single else 300)
        o["C"].fill_(7.0)
        S.run(shapes, b, o)  # eagerly: the same bits
        torch.cuda.synchronize()
        assert torch.equal(o["C"], got)
    N.ntp_destroy(S.h)


def test_two_streams_with_handles_of_their_own():
    import torch
    import paper_2504_06095_amd as N
    servers = [Server([900, 500], 16, 2, 128, 8, 0, 32, 8, seed=11 + i) for i in range(2)]
    jobs = []
    for S, news in zip(servers, ((900, 500), (600, 1))):
        rows = sum(news)
        shapes, b, o = S.shapes(rows, 900), S.batch(news, rows), S.buffers(rows)
        if shapes[2]:
            N.ntp_set_workspace(torch.empty(shapes[2], dtype=torch.uint8, device="cuda"), handle=S.h)
        S.run(shapes, b, o)
        torch.cuda.synchronize()
        jobs.append((S, shapes, b, o, o["C"].clone()))
    streams = [torch.cuda.Stream() for _ in jobs]
    for _ in range(4):
        for job in jobs:
            job[3]["C"].fill_(7.0)
        torch.cuda.synchronize()
        for st, (S, shapes, b, o, _) in zip(streams, jobs):
            with torch.cuda.stream(st):
                S.run(shapes, b, o)
                S.run(shapes, b, o)
        torch.cuda.synchronize()
        for S, shapes, b, o, want in jobs:
            assert torch.equal(o["C"], want)
    for S in servers:
        N.ntp_destroy(S.h)


@pytest.mark.parametrize("d", [64, 128])
def test_the_gradient_goes_through_the_core_and_the_norms(d):
    """Forward: norms and rotation inside QKV's copy, attention core; backward: the core's dQKV, then the norms' gradient in its place."""
    import torch
    import paper_2504_06095_amd as N
    n_seq, S = 2, 150
    plan, M = N.ntp_attn_shard_plan(8, 2, d, 3, 0), 2 * 150
    q, kv, wq, wk = plan["q_cnt"], plan["kv_cnt"], plan["q_cnt"] * d, plan["kv_cnt"] * d
    g = torch.Generator(device="cuda").manual_seed(d)
    raw = torch.randn(M, plan["w_qkv"], device="cuda", generator=g).bfloat16()
    gq, gk = ((1 + 0.2 * torch.randn(d, device="cuda", generator=g)).bfloat16() for _ in range(2))
    norm, shape = N.qk_norm(gq, gk, EPS), N.kv_append_shape(M, plan)
    f = torch.tensor([10000.0 ** (-2 * i / d) for i in range(d // 2)], dtype=torch.float64, device="cuda")
    pos = torch.arange(S, dtype=torch.int32, device="cuda").repeat(n_seq)
    QKV = raw.clone()
    N.ntp_qk_norm_append_shard(shape, norm, None, raw, pos, None, f, QKV[:, :wq], QKV[:, wq:wq + wk])
    core = N.attn_core_shape(n_seq, S, plan, 4, True)
    C, dC = (torch.randn(M, wq, device="cuda", generator=g).bfloat16() for _ in range(2))
    LSE, Delta, dQKV = torch.empty(q, M, device="cuda"), torch.empty(q, M, device="cuda"), torch.empty_like(QKV)
    N.ntp_attn_core_shard_fwd(core, QKV, C, LSE)
    N.ntp_attn_core_shard_bwd(core, QKV, C, dC, LSE, Delta, dQKV)
    torch.cuda.synchronize()
    up = dQKV.clone()
    da, db = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    N.ntp_qk_norm_shard_bwd(shape, norm, raw, dQKV[:, :wq], dQKV[:, wq:wq + wk], pos, f, dQKV, da, db)
    torch.cuda.synchronize()
    p = pos.cpu().numpy()
    wQ, wK, _ = B.qk_norm(f64(raw), q, kv, d, f64(gq), f64(gk), EPS, p, f.cpu().numpy(), False)
    assert np.abs(f64(QKV[:, :wq]) - wQ.reshape(M, -1)).max() <= 2 * BF * np.abs(wQ).max() and np.abs(f64(QKV[:, wq:wq + wk]) - wK.reshape(M, -1)).max() <= 2 * BF * np.abs(wK).max()
    want, wa, wb = B.qk_norm_bwd(f64(raw), q, kv, d, f64(gq), f64(gk), EPS, p, f.cpu().numpy(), False, f64(up[:, :wq]), f64(up[:, wq:wq + wk]))
    assert np.abs(f64(dQKV[:, :wq + wk]) - want).max() <= 2 * BF * np.abs(want).max()
    assert torch.equal(dQKV[:, wq + wk:], up[:, wq + wk:])
    for got, ref in ((da, wa), (db, wb)):
        assert np.abs(f64(got) - ref).max() <= 1e-4 * np.abs(ref).max()
